// Orthogonalised updates (Muon) for sm_103a: momentum, Newton-Schulz steps, the weights' update.
//
// A Newton-Schulz step takes a matrix X, n its smaller side, to p(A) X with A = X X^T and
// p(t) = a + b t + c t^2 (a tall X: to X p(X^T X)): every singular value s goes to s p(s^2), which with
// Muon's coefficients brings it near 1 from anywhere in (0, 1] in about five steps.  With X scaled to
// Frobenius norm 1 first,
//
//   k_muon_first   m = mu m + d, and the sum of squares of what is orthogonalised, a part a tile
//   k_muon_scale   X = u / |u|, in fp16
//   k_product      A = X X^T;  B = a I + b A + c A^2;  X' = B X: three launches a step.  The last one writes
//                  the weights and their copies, or the values themselves
//   k_muon_last    does that for matrices whose rows do not lie on 32-byte boundaries
//   k_gram_sum     A of matrices with a side beyond 65536, whose sums are taken in parts
//   k_muon_small   all of it for matrices that a CTA's shared memory holds
//
// One launch covers all matrices of a list.  The products are nearly all of the work: per step 2 n^2 m and
// 2 n^3 operations of which symmetry leaves half, and 2 n^2 m.  They run on the tensor cores from fp16
// operands with fp32 sums.  Why fp16: all values are bounded (singular values of at most about 1.2, so
// elements too), and its 11 bits leave the result 1 to 2e-3 off, where bf16's 8 leave it 1e-2 off, for singular values
// within 20 of the largest (a rounding of 2^-12 of that falls on the others and grows with them by up to 3.4445 a step:
// 2e-2 for values that fall off like 1 / k^2, where rounding the matrix itself to bf16 moves the result by 0.15); the
// first step's X, whose elements are about 1 / sqrt(n m), is kept larger by a power of two.  B takes in a I before
// it is rounded: then its diagonal is near 0.7 instead of -2.7, and X need not be added afterwards.
//
// Matrices lie in the workspace as tiles of 128 rows by 64 columns, 16 KB each, zero beyond the matrix, and
// the whole workspace is one array of 128-byte rows to the copies: a tile is 128 of them.  Brought to shared
// memory with the 128-byte swizzle, its rows serve as an operand with the sum along the tile's columns or
// along its rows (the instruction's K- or MN-major forms have the same image), so nothing is ever transposed
// in memory: X is read both ways, and tall matrices stay as they are.
#include "tula_tc.cuh"

#include <cmath>
#include <memory>
#include <new>
#include <vector>

namespace {

constexpr double kA = 3.4445, kB = -4.7750, kC = 2.0315;
constexpr int kTileCols = 64, kTileBytes = kTile * 128;
constexpr int kMostGroups = 32;    // shapes of one launch
constexpr int kMostSteps = 100;
constexpr long long kMostSide = 1LL << 20;
constexpr long long kMostTiles = 1LL << 24;  // of a workspace: rows of 128 bytes fit an int
// Elements that A's sums run over at a time.  The tensor cores cut their fp32 sums off, 16 products at a time, so that
// a sum of squares loses up to 2^-23 of itself with each: O of 2^20 x 1 was 5e-3 off with one sum, three times what
// fp16 operands leave.  Parts are rounded to fp16 and added in fp32, which costs less than the sum's own rounding.
constexpr int kMostSum = 65536;

// ----------------------------------------------------------------------------
// Products
// ----------------------------------------------------------------------------

// An operand of 128 (or 256, by pairs) rows of the product's side: in tiles of `pitch` to a row of them.  The sum
// runs along the tiles' columns (K-major) or along their rows; of a symmetric matrix, of which the blocks on
// and above the diagonal are there, along rows up to the diagonal and along columns from there on.  (With the
// blocks below it written too, transposed by way of shared memory, 8192 x 8192 took 6.59 ms instead of 6.36 and
// 1024 x 1024 178 us instead of 162.)
enum Way { kAcross, kAlong, kSymmetric };
struct Side {
    int base, step;   // the first matrix's first tile, tiles from matrix to matrix
    int pitch, rows;  // tiles
    int way;
    // The first stage that runs along the columns, of the operand of block `block` of kSide.  (Symmetric ones are
    // there by blocks of 256, whatever kSide made them.)
    template <int kSide>
    __device__ __forceinline__ int turn(int block) const {
        return way == kAlong ? 0 : way == kAcross ? 1 << 30 : block * kSide / 256 * 4;
    }
};
struct Matrix {  // of a plan
    const void *g;
    float *m, *w;
    void *copy;
    int gtype, ctype, vec, spare;  // vec: elements of a row at a time, see load_tile
};
struct ProductGroup {
    Side p, q;
    int out, out_step, out_pitch, out_rows;
    int first, per;   // the group's first block of work, blocks to a matrix
    int blocks_m, blocks_n;
    int n_k;          // stages of 64
    int n;            // where the identity ends
    float alpha;
    int finish;       // kLast: the weights or values are written
    int rows, cols, matrix;  // the first one's place in the plan's table
    float step;       // lr times the shape's factor
};
struct ProductArgs {
    const unsigned char *tiles;
    const float *record;
    const Matrix *matrices;  // kLast: a plan's, or NULL:
    void *y;                 // the values' place, contiguous
    int ytype;
    float decay;
    int n_groups, n_blocks;
    int n_first, skip;  // see block_of
    int none;         // a row beyond the workspace
    ProductGroup g[kMostGroups];
};
static_assert(sizeof(ProductArgs) <= 4096 - 2 * 128 - 64, "kernel parameters");

// What is made of the sums: alpha times them, of a symmetric product (its blocks on and above the diagonal are
// taken); the polynomial, symmetric too; alpha times them; the same of the last step, which
// goes straight to the weights.  (HBM bounds that: 359 us for 151 M weights in place of 176 and 299 one after the
// other.)
enum Kind { kGram, kPoly, kApply, kLast };

// A copying warp, an issuing warp, and those that read back: two to each quarter of tensor memory's lanes, each
// with half of the columns (72 matrices of 151 M elements, most sums of 1024: 2.66 to 2.71 ms, 2.72 to 2.78 with one
// to a quarter).
constexpr int kReaders = 8;
constexpr int kThreads = 64 + 32 * kReaders;

template <bool Pair>
struct Shape {
    static constexpr int kSide = Pair ? 256 : 128;  // of a block of the output
    static constexpr int kStages = 6;  // (what is on its way bounds the rate: X' of 151 M in 176 us, 184 with five)
    static constexpr int kOperand = 128 * 128;      // bytes of a stage, a CTA
    static constexpr int kStage = 2 * kOperand;
    static constexpr int kOuts = kReaders * 4096;   // a buffer a warp
    static constexpr int kBars = 2 * kStages + 4;
    static constexpr int kSmem = kStages * kStage + kOuts + 8 * kBars + 16 + 1024;
    static constexpr int kCols = 2 * kSide;         // two accumulators
    static_assert(kSmem <= 227 * 1024, "shared memory");
};
// Shared-memory matrix descriptors of an operand (bit 46: their version; the 128-byte swizzle).  Along: rows of
// 64 elements of the sum, groups of eight 1024 bytes apart.  Else: rows of 64 of the side, one for each element
// of the sum, groups of eight 1024 bytes apart, the next 64 of the side `next` bytes on.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool along, unsigned next = 8192) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(along ? 1 : next >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// fp16 operands, fp32 sums.
__device__ __forceinline__ uint32_t product_desc(int m, int n, bool p_along, bool q_along) {
    return 1u << 4 | (p_along ? 0u : 1u << 15) | (q_along ? 0u : 1u << 16) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
template <bool Pair>
__device__ __forceinline__ void mma16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if (Pair)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
                     : "memory");
}

// The blocks in the order of their groups, those with the longest sums first, go round the workers; those that
// the first groups, of equal sums, leave with one more than the others are passed over for a.skip rounds of what follows, about
// as long as that one takes.  (72 matrices, sums of 4096 and of 1024: A in 108 us, 119 without.)
__device__ __forceinline__ int block_of(const ProductArgs &a, int worker, int workers, int i) {
    const int full = a.n_first / workers, more = a.n_first - full * workers;
    if (i < full) return i * workers + worker;
    if (!a.skip) return i * workers + worker;
    i -= full;
    const bool heavy = worker < more;
    if (heavy && i == 0) return full * workers + worker;
    if (!heavy && i < a.skip) return a.n_first + i * (workers - more) + worker - more;
    return a.n_first + a.skip * (workers - more) + (i - (heavy ? 1 : a.skip)) * workers + worker;
}

// A block of work: its group, matrix and place.
struct Block {
    int matrix, m, n;
};
// A symmetric product's blocks in column n: those on and above the diagonal, by 256.
template <int kSide>
__host__ __device__ constexpr int column_blocks(int n, int blocks) {
    return kSide == 256 ? n + 1 : (n | 1) + 1 < blocks ? (n | 1) + 1 : blocks;
}
template <Kind K, int kSide>
__device__ __forceinline__ Block block_at(const ProductArgs &a, int t, const ProductGroup *&g) {
    int i = 0;
    while (i + 1 < a.n_groups && t >= a.g[i + 1].first) ++i;
    g = &a.g[i];
    const int in = t - g->first;
    Block b;
    b.matrix = in / g->per;
    int k = in - b.matrix * g->per;
    if (K >= kApply) {
        b.m = k % g->blocks_m;
        b.n = k / g->blocks_m;
    } else {
        b.n = 0;
        while (k >= column_blocks<kSide>(b.n, g->blocks_n)) k -= column_blocks<kSide>(b.n++, g->blocks_n);
        b.m = k;
    }
    return b;
}

// Rows of the workspace that an operand's stages start at, in registers: the loops are full of statements that
// the compiler may not move loads across, and with the group's fields read again for each stage the copying
// warp took some 800 cycles to one.
struct Walk {
    unsigned row0, row1;      // of the two halves of a stage; none where there are none
    unsigned odd, even;       // rows from an even stage to the odd one after it, and from there to the next
    unsigned along0, along1;  // of stage `turn`
    int turn;
    __device__ __forceinline__ Walk(const Side &s, int matrix, int i, int first_along, unsigned none) : turn(first_along) {
        const int first = s.base + matrix * s.step;
        along0 = i < s.rows ? (first + i * s.pitch + (turn < s.pitch ? turn : 0)) * kTile : none;
        along1 = along0 == none ? none : along0 + 64;
        row0 = 2 * i < s.pitch ? (first + 2 * i) * kTile : none;
        row1 = 2 * i + 1 < s.pitch ? (first + 2 * i + 1) * kTile : none;
        odd = 64;
        even = s.pitch * kTile - 64;
        if (turn == 0) columns();
        // (none and what comes after it lie beyond the workspace, also as negative coordinates)
    }
    __device__ __forceinline__ void columns() {
        row0 = along0;
        row1 = along1;
        odd = even = kTile;
    }
    __device__ __forceinline__ void next(int k) {
        const unsigned by = k & 1 ? even : odd;
        row0 += by;
        row1 += by;
        if (k + 1 == turn) columns();
    }
};

// Eight elements on a boundary of 32 bytes (fp32) or 16.
__device__ __forceinline__ void load8(float *f, const float *from) {
    unsigned r[8];
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(from));
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void store8(float *to, const float (&f)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(__float_as_uint(f[0])),
                 "r"(__float_as_uint(f[1])), "r"(__float_as_uint(f[2])), "r"(__float_as_uint(f[3])), "r"(__float_as_uint(f[4])),
                 "r"(__float_as_uint(f[5])), "r"(__float_as_uint(f[6])), "r"(__float_as_uint(f[7]))
                 : "memory");
}
__device__ __forceinline__ void store8(void *to, int type, size_t at, const float (&f)[8]) {
    unsigned u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (type == TULA_TYPE_BF16) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
            memcpy(&u[k], &h, 4);
        } else {
            const __half2 h = __floats2half2_rn(f[2 * k], f[2 * k + 1]);
            memcpy(&u[k], &h, 4);
        }
    }
    *reinterpret_cast<uint4 *>(static_cast<unsigned short *>(to) + at) = make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

template <bool Pair, Kind K>
__global__ void __launch_bounds__(kThreads, 1)
    k_product(const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_out,
              const __grid_constant__ ProductArgs a) {
    using S = Shape<Pair>;
    extern __shared__ __align__(16) unsigned char raw[];
    unsigned char *all = raw + (-smem_addr(raw) & 1023u);
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(all + S::kStages * S::kStage + S::kOuts);
    uint32_t *tmem_at = reinterpret_cast<uint32_t *>(bars + S::kBars);
    volatile int &dead = *reinterpret_cast<volatile int *>(tmem_at + 1);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFull, tid >> 5, 0);
    const unsigned rank = Pair ? blockIdx.x & 1 : 0;
    const int workers = Pair ? gridDim.x / 2 : gridDim.x, worker = Pair ? blockIdx.x / 2 : blockIdx.x;
    const uint32_t stages = smem_addr(all), outs = stages + S::kStages * S::kStage;
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, acc_free = acc_full + 16;
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full + 8 * s, 1);
            mbar_init(acc_free + 8 * s, (Pair ? 2 : 1) * kReaders);  // the reading warps, of both CTAs
        }
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && elect_one()) prefetch_map(&map_in);
    if (warp == 2 && elect_one()) prefetch_map(&map_out);
    if (warp == 1) {
        if (Pair) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_at)), "r"(S::kCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            tmem_alloc(smem_addr(tmem_at), S::kCols);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (Pair) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(kFull, *tmem_at, 0);
    let_next_start();
    // Each role goes through its loop once before it waits for the kernel ahead, without what the others or memory
    // would see of it: so its instructions and the first block's parameters are there when the wait ends.  (1024 x
    // 1024: 162 us without, 153 so.)
    auto blocks_after_wait = [&] {
        wait_for_previous();
        return !a.record || a.record[TULA_RECORD_FINITE] != 0.f ? a.n_blocks : 0;
    };
    int n_blocks = 0;

    if (warp == 0) {
        int i = 0;  // stages filled
        bool ok = true, dry = true;
#pragma unroll 1
        for (int at_block = 0; ok;) {
            int t = block_of(a, worker, workers, at_block);
            if (dry)
                t = min(t, a.n_blocks - 1);
            else if (t >= n_blocks)
                break;
            const ProductGroup *g;
            const Block b = block_at<K, S::kSide>(a, t, g);
            const int n_k = dry ? 1 : g->n_k;
            Walk p(g->p, b.matrix, Pair ? 2 * b.m + rank : b.m, g->p.turn<S::kSide>(b.m), a.none);
            Walk q(g->q, b.matrix, Pair ? 2 * b.n + rank : b.n, g->q.turn<S::kSide>(b.n), a.none);
#pragma unroll 1
            for (int k = 0; k < n_k; ++k) {
                const int s = i % S::kStages;
                if (i >= S::kStages) ok = __all_sync(kFull, mbar_wait(empty + 8 * s, (i / S::kStages - 1) & 1, &dead));
                if (!ok) break;
                const uint32_t at = stages + s * S::kStage, bar = Pair ? in_cta(full + 8 * s, 0) : full + 8 * s;
                if (elect_one() && !dry) {
                    if (rank == 0) mbar_expect(full + 8 * s, (Pair ? 2 : 1) * S::kStage);  // both CTAs' copies
                    if (Pair) {
                        tma_load_pair(at, &map_in, 0, (int)p.row0, bar);
                        tma_load_pair(at + 8192, &map_in, 0, (int)p.row1, bar);
                        tma_load_pair(at + S::kOperand, &map_in, 0, (int)q.row0, bar);
                        tma_load_pair(at + S::kOperand + 8192, &map_in, 0, (int)q.row1, bar);
                    } else {
                        tma_load_2d(at, &map_in, 0, (int)p.row0, bar);
                        tma_load_2d(at + 8192, &map_in, 0, (int)p.row1, bar);
                        tma_load_2d(at + S::kOperand, &map_in, 0, (int)q.row0, bar);
                        tma_load_2d(at + S::kOperand + 8192, &map_in, 0, (int)q.row1, bar);
                    }
                }
                __syncwarp();
                p.next(k);
                q.next(k);
                if (!dry) ++i;
            }
            if (dry) {
                dry = false;
                n_blocks = blocks_after_wait();
            } else {
                ++at_block;
            }
        }
        // The issuing warp's arrivals (of the other CTA too) have all landed before the CTA ends.
        for (int j = max(0, i - S::kStages); ok && j < i; ++j)
            ok = __all_sync(kFull, mbar_wait(empty + 8 * (j % S::kStages), (j / S::kStages) & 1, &dead));
        // No copy may be in flight when the CTA ends.  On the way out of a wait that ran out
        // the copies' barrier may be the other CTA's: a millisecond is far more than they take.
        if (!ok)
            for (int w = 0; w < 1000; ++w) __nanosleep(1000);
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            int i = 0, n = 0;
            bool ok = true, dry = true;
#pragma unroll 1
            for (; ok;) {
                int t = block_of(a, worker, workers, n);
                if (dry)
                    t = min(t, a.n_blocks - 1);
                else if (t >= n_blocks)
                    break;
                const ProductGroup *g;
                const Block b = block_at<K, S::kSide>(a, t, g);
                const int n_k = dry ? 1 : g->n_k, p_turn = g->p.turn<S::kSide>(b.m), q_turn = g->q.turn<S::kSide>(b.n);
                if (n > 1) ok = __all_sync(kFull, mbar_wait(acc_free + 8 * (n & 1), (n / 2 - 1) & 1, &dead));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t acc = tmem + (n & 1) * S::kSide;
#pragma unroll 1
                for (int k = 0; ok && k < n_k; ++k) {
                    const int s = i % S::kStages;
                    if (!dry) ok = __all_sync(kFull, mbar_wait(full + 8 * s, (i / S::kStages) & 1, &dead));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = stages + s * S::kStage;
                    const bool pa = k >= p_turn, qa = k >= q_turn;
                    const uint32_t idesc = product_desc(S::kSide, S::kSide, pa, qa);
                    // from one instruction's 16 of the sum to the next: 32 bytes of a row, or 16 rows
                    const uint32_t p_next = pa ? 2 : 128, q_next = qa ? 2 : 128;
                    const uint64_t dp = operand_desc(at, pa), dq = operand_desc(at + S::kOperand, qa);
                    if (elect_one() && !dry) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma16<Pair>(acc, dp + j * p_next, dq + j * q_next, idesc, k > 0 || j > 0);
                        if (Pair) {
                            commit_pair(empty + 8 * s);
                            if (k == n_k - 1) commit_pair(acc_full + 8 * (n & 1));
                        } else {
                            commit(empty + 8 * s);
                            if (k == n_k - 1) commit(acc_full + 8 * (n & 1));
                        }
                    }
                    __syncwarp();
                    if (!dry) ++i;
                }
                if (dry) {
                    dry = false;
                    n_blocks = blocks_after_wait();
                } else {
                    ++n;
                }
            }
        } else {
            wait_for_previous();
        }
        __syncwarp();
    } else {
        const int quad = warp & 3, row = quad * 32 + lane, half = (warp - 2) >> 2;
        constexpr int kChunks = S::kSide / kTileCols / (kReaders / 4);  // of 64 columns, a warp
        const uint32_t buffer = outs + (warp - 2) * 4096;
        auto buffer_free = [&] {  // the store that last used it has read it
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
        };
        int n = 0;
        bool dry = true;
#pragma unroll 1
        for (;;) {
            int t = block_of(a, worker, workers, n);
            if (dry)
                t = min(t, a.n_blocks - 1);
            else if (t >= n_blocks)
                break;
            const ProductGroup *g;
            const Block b = block_at<K, S::kSide>(a, t, g);
            const int im = Pair ? 2 * b.m + rank : b.m;
            const int out = g->out + b.matrix * g->out_step;
            const int j0 = b.n * (S::kSide / kTileCols) + half * kChunks;  // column of tiles
            const int out_pitch = g->out_pitch;
            const int chunks = im < g->out_rows ? max(0, min(kChunks, out_pitch - j0)) : 0;  // within the output
            const float alpha = g->alpha, step = g->step;
            // kPoly: A's rows come to the buffer, each lane's own, and B takes their place there
            const unsigned char *const added =
                a.tiles + (size_t)(g->p.base + b.matrix * g->p.step + im * g->p.pitch + j0) * kTileBytes + row * 128;
            auto fetch = [&](int c) {
                buffer_free();
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(buffer + lane * 128 + ((k ^ (lane & 7)) << 4)),
                                 "l"(added + (size_t)c * kTileBytes + 16 * k)
                                 : "memory");
            };
            if (K == kPoly && chunks && !dry) fetch(0);
            const bool finish = K == kLast && g->finish;
            if (!dry && !__all_sync(kFull, mbar_wait(acc_full + 8 * (n & 1), (n / 2) & 1, &dead))) {
                if (K == kPoly) asm volatile("cp.async.wait_all;" ::: "memory");
                break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + (n & 1) * S::kSide + half * kChunks * kTileCols + ((unsigned)(quad * 32) << 16);
            if constexpr (K == kLast) {
                if (finish) {
                    // the weights move by four lanes to 32 columns of a row
                    const int first_row = im * kTile + quad * 32 + (lane >> 2), cols = g->cols, rows_left = dry ? 0 : g->rows - first_row;
                    Matrix q = {};
                    if (a.matrices && !dry) q = a.matrices[g->matrix + b.matrix];
                    buffer_free();  // (of a block of another group)
#pragma unroll 1
                    for (int c = 0; c < chunks; ++c) {
                        const int col = (j0 + c) * kTileCols + (lane & 3) * 8;  // and 32 further on
                        unsigned v[64];
                        tmem_load32(v, acc + c * kTileCols);
                        tmem_load32(v + 32, acc + c * kTileCols + 32);
                        float w[64];
                        if (q.w) {
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (8 * (k & 3) < rows_left && col + 8 * (k & 4) < cols)
                                    load8(w + 8 * k, q.w + (size_t)(first_row + 8 * (k & 3)) * cols + col + 8 * (k & 4));
                        }
                        tmem_wait(v);
                        // the values change from a row a lane to a row four lanes, 32 rows of 32 columns at a
                        // time, their 32-byte pieces exchanged so that neither way meets in a bank
#pragma unroll
                        for (int half_at = 0; half_at < 2; ++half_at) {
                            __syncwarp();  // the last ones have been read
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                                 buffer + lane * 128 + ((k ^ (lane & 3) << 1) << 4)),
                                             "r"(v[32 * half_at + 4 * k]), "r"(v[32 * half_at + 4 * k + 1]),
                                             "r"(v[32 * half_at + 4 * k + 2]), "r"(v[32 * half_at + 4 * k + 3])
                                             : "memory");
                            __syncwarp();
                            const int c0 = col + 32 * half_at;
                            if (c0 < cols) {
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    if (8 * k >= rows_left) break;
                                    const int r = 8 * k + (lane >> 2);
                                    const uint32_t from = buffer + r * 128 + (((lane & 3) ^ (r & 3)) << 5);
                                    float x[8];
#pragma unroll
                                    for (int h = 0; h < 2; ++h)
                                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                                                     : "=f"(x[4 * h]), "=f"(x[4 * h + 1]), "=f"(x[4 * h + 2]), "=f"(x[4 * h + 3])
                                                     : "r"(from + 16 * h)
                                                     : "memory");
#pragma unroll
                                    for (int e = 0; e < 8; ++e) x[e] *= alpha;
                                    const size_t at = (size_t)(first_row + 8 * k) * cols + c0;
                                    if (q.w) {
#pragma unroll
                                        for (int e = 0; e < 8; ++e)
                                            x[e] = fmaf(-step, x[e], __fmul_rn(w[32 * half_at + 8 * k + e], a.decay));
                                        store8(q.w + at, x);
                                        if (q.copy) store8(q.copy, q.ctype, at, x);
                                    } else {
                                        store8(a.y, a.ytype, (size_t)b.matrix * g->rows * cols + at, x);
                                    }
                                }
                            }
                        }
                    }
                }
            }
#pragma unroll 1
            for (int c = 0; c < chunks && !finish; ++c) {
                if (K != kPoly)
                    buffer_free();
                else if (c && !dry)
                    fetch(c);
                const int diagonal = im * kTile + row < g->n ? im * kTile + row - (j0 + c) * kTileCols : -1;
                unsigned v[64];
                tmem_load32(v, acc + c * kTileCols);
                tmem_load32(v + 32, acc + c * kTileCols + 32);
                if (K == kPoly) asm volatile("cp.async.wait_all;" ::: "memory");
                tmem_wait(v);
#pragma unroll
                for (int h = 0; h < 8; ++h) {  // eight columns
                    const uint32_t at = buffer + lane * 128 + ((h ^ (lane & 7)) << 4);
                    float f[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(v[8 * h + k]);
                    if (K == kPoly) {
                        unsigned add[4];
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(add[0]), "=r"(add[1]), "=r"(add[2]), "=r"(add[3])
                                     : "r"(at)
                                     : "memory");
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            __half2 e;
                            memcpy(&e, &add[k], 4);
                            const float2 x = __half22float2(e);
                            f[2 * k] = fmaf((float)kC, f[2 * k], fmaf((float)kB, x.x, diagonal == 8 * h + 2 * k ? (float)kA : 0.f));
                            f[2 * k + 1] = fmaf((float)kC, f[2 * k + 1], fmaf((float)kB, x.y, diagonal == 8 * h + 2 * k + 1 ? (float)kA : 0.f));
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] *= alpha;
                    }
                    unsigned y[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const __half2 e = __floats2half2_rn(f[2 * k], f[2 * k + 1]);
                        memcpy(&y[k], &e, 4);
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0 && !dry)
                    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];\n"
                                 "cp.async.bulk.commit_group;" ::"l"(&map_out),
                                 "r"(0), "r"((out + im * out_pitch + j0 + c) * kTile + quad * 32), "r"(buffer)
                                 : "memory");
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (dry) {
                dry = false;
                n_blocks = blocks_after_wait();
                continue;
            }
            if (lane == 0) arrive_cluster(Pair ? in_cta(acc_free + 8 * (n & 1), 0) : acc_free + 8 * (n & 1));
            ++n;
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (Pair) cluster_sync();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (Pair)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kCols));
        else
            tmem_free(tmem, S::kCols);
    }
}

// ----------------------------------------------------------------------------
// Before and after the products
// ----------------------------------------------------------------------------
//
// One CTA a tile of 128 x 64, 32 elements a thread, V of a row at a time: eight where all buffers' rows have a
// multiple of eight at boundaries of 16 bytes, two where they have an even number at boundaries of two (6 of
// 4099 x 1502 bf16: 110 us for the three kernels, 149 one by one and three CTAs an SM), else one.  These stream: 8 to 22 bytes an
// element.

struct Group {
    int first, per;       // the group's first tile of all, tiles to a matrix
    int matrix;           // its first matrix
    int rows, cols, pitch;  // pitch: tiles to a row of tiles
    int x, x_last;        // X's first tile, and the last step's
    float scale;          // the power of two that X is larger by at first
    float step;           // lr times the shape's factor
};
struct StreamArgs {
    const Matrix *matrices;  // a plan's, or NULL: one group,
    const void *x;           // read from here
    long long stride, batch_stride;
    void *y;                 // and written there, contiguous
    int xtype, ytype, vec;
    unsigned char *tiles;
    double *parts;           // sums of squares, one a tile
    const float *record;
    float grad_scale, mu, decay;
    int nesterov, n_groups, tile0;  // tile0: k_muon_last's first
    Group g[kMostGroups];
};
static_assert(sizeof(StreamArgs) <= 4096 - 64, "kernel parameters");

constexpr int kStreamThreads = 256;
// CTAs an SM, that registers are left for: of a plan's matrices, which have a momentum or weights to hold too, and
// of others (with three for both, 145 us for those; k_muon_scale has four, at five it spills).
template <bool Plan>
constexpr int kStreamCtas = Plan ? 3 : 5;

struct Place {
    const Group *g;
    int matrix, tile;      // of the group, of the matrix
    int row0, col0;
};
__device__ __forceinline__ Place place_of(const StreamArgs &a, int t) {
    int i = 0;
    while (i + 1 < a.n_groups && t >= a.g[i + 1].first) ++i;
    Place p;
    p.g = &a.g[i];
    p.matrix = (t - p.g->first) / p.g->per;
    p.tile = t - p.g->first - p.matrix * p.g->per;
    p.row0 = p.tile / p.g->pitch * kTile;
    p.col0 = p.tile % p.g->pitch * kTileCols;
    return p;
}
// Element k of a thread's 32, within the tile.
template <int V>
__device__ __forceinline__ int row_of(int k) { return k / V * (4 * V) + threadIdx.x / (kTileCols / V); }
template <int V>
__device__ __forceinline__ int col_of(int k) { return threadIdx.x % (kTileCols / V) * V + k % V; }

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float value(__half v) { return __half2float(v); }

template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Run {
    T v[N];
};
// A thread's elements of a matrix whose rows lie `stride` apart; zero beyond it.
template <typename T, int V>
__device__ __forceinline__ void load_tile(float (&f)[32], const T *base, long long stride, const Place &p) {
    constexpr int kN = V;
    Run<T, kN> r[32 / kN];
#pragma unroll
    for (int k = 0; k < 32; k += kN) {
        const int i = p.row0 + row_of<V>(k), j = p.col0 + col_of<V>(k);
        if (i < p.g->rows && j < p.g->cols)
            r[k / kN] = *reinterpret_cast<const Run<T, kN> *>(base + i * stride + j);
        else
#pragma unroll
            for (int e = 0; e < kN; ++e) r[k / kN].v[e] = T(0.f);
    }
#pragma unroll
    for (int k = 0; k < 32; ++k) f[k] = value(r[k / kN].v[k % kN]);
}
template <typename T, int V>
__device__ __forceinline__ void store_tile(T *base, long long stride, const Place &p, const float (&f)[32]) {
    constexpr int kN = V;
#pragma unroll
    for (int k = 0; k < 32; k += kN) {
        const int i = p.row0 + row_of<V>(k), j = p.col0 + col_of<V>(k);
        if (i >= p.g->rows || j >= p.g->cols) continue;
        Run<T, kN> r;
#pragma unroll
        for (int e = 0; e < kN; ++e) put(&r.v[e], f[k + e]);
        *reinterpret_cast<Run<T, kN> *>(base + i * stride + j) = r;
    }
}
template <int V>
__device__ __forceinline__ void load_typed(float (&f)[32], const void *base, int type, long long stride, const Place &p) {
    if (type == TULA_TYPE_F32)
        load_tile<float, V>(f, static_cast<const float *>(base), stride, p);
    else if (type == TULA_TYPE_BF16)
        load_tile<__nv_bfloat16, V>(f, static_cast<const __nv_bfloat16 *>(base), stride, p);
    else
        load_tile<__half, V>(f, static_cast<const __half *>(base), stride, p);
}
template <int V>
__device__ __forceinline__ void store_typed(void *base, int type, long long stride, const Place &p, const float (&f)[32]) {
    if (type == TULA_TYPE_BF16)
        store_tile<__nv_bfloat16, V>(static_cast<__nv_bfloat16 *>(base), stride, p, f);
    else
        store_tile<__half, V>(static_cast<__half *>(base), stride, p, f);
}
// A plan's element type starts at the matrix; another's matrices lie batch_stride apart.
__device__ __forceinline__ const void *batch_at(const StreamArgs &a, int matrix) {
    return static_cast<const unsigned char *>(a.x) + (size_t)matrix * a.batch_stride * (a.xtype == TULA_TYPE_F32 ? 4 : 2);
}

// What is orthogonalised: its parts as they lie in memory, and then the update itself.  First: the momentum
// moves on.
template <bool Plan>
struct Loaded {
    float g[32], m[Plan ? 32 : 1], mult;
};
template <bool Plan, int V>
__device__ __forceinline__ void load_parts(Loaded<Plan> &l, const StreamArgs &a, const Place &p, const Matrix &q) {
    if constexpr (Plan) {
        l.mult = a.record ? __fdiv_rn(a.record[TULA_RECORD_COEF], a.grad_scale) : __fdiv_rn(1.f, a.grad_scale);
        load_typed<V>(l.g, q.g, q.gtype, p.g->cols, p);
        load_tile<float, V>(l.m, q.m, p.g->cols, p);
    } else {
        load_typed<V>(l.g, batch_at(a, p.matrix), a.xtype, a.stride, p);
    }
}
template <bool First, bool Plan, int V>
__device__ __forceinline__ void update_of(float (&u)[32], Loaded<Plan> &l, const StreamArgs &a, const Place &p, const Matrix &q) {
    if constexpr (Plan) {
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            const float d = __fmul_rn(l.g[k], l.mult);
            if (First) l.m[k] = fmaf(a.mu, l.m[k], d);
            u[k] = a.nesterov ? fmaf(a.mu, l.m[k], d) : l.m[k];
        }
        if (First) store_tile<float, V>(q.m, p.g->cols, p, l.m);
    } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) u[k] = l.g[k];
    }
}
template <bool First, bool Plan, int V>
__device__ __forceinline__ void load_update(float (&u)[32], const StreamArgs &a, const Place &p, const Matrix &q) {
    Loaded<Plan> l;
    load_parts<Plan, V>(l, a, p, q);
    update_of<First, Plan, V>(u, l, a, p, q);
}

// The sum of squares of a warp's elements: in fp32 with an exact power of two taken out, so that no square
// leaves its range.
__device__ __forceinline__ void warp_squares(const float (&u)[32], double *sums) {
    unsigned top = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) top = max(top, __float_as_uint(u[k]) & 0x7fffffffu);
    top = __reduce_max_sync(kFull, top) >> 23;
    const unsigned e = min(top, 253u);
    const float f = __uint_as_float((254u - e) << 23);  // 2^(127 - e)
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        const float v = __fmul_rn(u[k], f);
        s = fmaf(v, v, s);
    }
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = (double)s * __hiloint2double((1023 + 2 * ((int)e - 127)) << 20, 0);
}

template <bool Plan, int V>
__device__ __forceinline__ void first_tile(const StreamArgs &a, const Place &p, const Matrix &q, double *sums) {
    float u[32];
    load_update<true, Plan, V>(u, a, p, q);
    warp_squares(u, sums);
}
__device__ __forceinline__ bool left_out(const StreamArgs &a) { return a.record && a.record[TULA_RECORD_FINITE] == 0.f; }

template <bool Plan>
__global__ void __launch_bounds__(kStreamThreads, kStreamCtas<Plan>) k_muon_first(const __grid_constant__ StreamArgs a) {
    __shared__ double sums[kStreamThreads / 32];
    let_next_start();
    wait_for_previous();
    if (left_out(a)) return;
    const Place p = place_of(a, blockIdx.x);
    Matrix q = {};
    if (Plan) q = a.matrices[p.g->matrix + p.matrix];
    switch (Plan ? q.vec : a.vec) {
        case 8: first_tile<Plan, 8>(a, p, q, sums); break;
        case 2: first_tile<Plan, 2>(a, p, q, sums); break;
        default: first_tile<Plan, 1>(a, p, q, sums);
    }
    __syncthreads();
    if (threadIdx.x) return;
    double s = 0.0;
    for (int k = 0; k < kStreamThreads / 32; ++k) s += sums[k];
    a.parts[blockIdx.x] = s;
}

// u / |u| as u f1 f2: f1 a power of two that brings u near 1, exactly, wherever in fp32's range it is.  A matrix of
// zeros stays, one with an infinity or NaN becomes NaN.  The norm is taken by every CTA for itself: one of
// its warps fetches the matrix's parts from L2 while the tile is on its way, one thread ends (an SM does
// some two fp64 operations a cycle: by all threads they took a third of the kernel's time).
__device__ __forceinline__ float2 factors_of(double squares, float scale) {
    if (!(squares < 1e300)) return make_float2(__uint_as_float(0x7fffffffu), __uint_as_float(0x7fffffffu));
    if (!(squares > 0.0)) return make_float2(0.f, 0.f);
    // |u| = root 2^k, 1 <= root < 2, in fp32 from here on
    const int k = ((int)((unsigned)__double2hiint(squares) >> 20) - 1023) >> 1;
    const float root = sqrtf((float)(squares * __hiloint2double((1023 - 2 * k) << 20, 0)));
    const int c = max(-126, min(126, k));
    return make_float2(__uint_as_float((unsigned)(127 - c) << 23), __fdiv_rn(scale, root) * __uint_as_float((unsigned)(127 + c - k) << 23));
}
__device__ __forceinline__ float2 norm_factors(const StreamArgs &a, const Place &p, float2 *factors) {
    if (threadIdx.x < 32) {
        const double *parts = a.parts + p.g->first + p.matrix * p.g->per;
        double s = 0.0;
        for (int i0 = 0; i0 < p.g->per; i0 += 256) {
            double v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + 32 * k + threadIdx.x;
                v[k] = i < p.g->per ? __ldcg(parts + i) : 0.0;
            }
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
        if (threadIdx.x == 0) {
            *factors = factors_of(s, p.g->scale);
        }
    }
    __syncthreads();
    return *factors;
}

// Elements of X from k on.
template <int V>
__device__ __forceinline__ Run<__half, V> scaled_run(const float (&u)[32], int k, const Place &p, float2 f) {
    Run<__half, V> r;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        // (a NaN factor leaves the zeros beyond the matrix alone)
        const bool in = p.row0 + row_of<V>(k + e) < p.g->rows && p.col0 + col_of<V>(k + e) < p.g->cols;
        r.v[e] = __float2half_rn(in ? __fmul_rn(__fmul_rn(u[k + e], f.x), f.y) : 0.f);
    }
    return r;
}
template <bool Plan, int V>
__device__ __forceinline__ void scale_tile(const StreamArgs &a, const Place &p, const Matrix &q, float2 *factors) {
    float u[32];
    load_update<false, Plan, V>(u, a, p, q);
    const float2 f = norm_factors(a, p, factors);
    __half *x = reinterpret_cast<__half *>(a.tiles + (size_t)(p.g->x + p.matrix * p.g->per + p.tile) * kTileBytes);
    constexpr int kN = V;
#pragma unroll
    for (int k = 0; k < 32; k += kN)
        *reinterpret_cast<Run<__half, kN> *>(x + row_of<V>(k) * kTileCols + col_of<V>(k)) = scaled_run<V>(u, k, p, f);
}
template <bool Plan>
__global__ void __launch_bounds__(kStreamThreads, Plan ? 3 : 4) k_muon_scale(const __grid_constant__ StreamArgs a) {
    __shared__ float2 factors;
    let_next_start();
    wait_for_previous();
    if (left_out(a)) return;
    const Place p = place_of(a, blockIdx.x);
    Matrix q = {};
    if (Plan) q = a.matrices[p.g->matrix + p.matrix];
    switch (Plan ? q.vec : a.vec) {
        case 8: scale_tile<Plan, 8>(a, p, q, &factors); break;
        case 2: scale_tile<Plan, 2>(a, p, q, &factors); break;
        default: scale_tile<Plan, 1>(a, p, q, &factors);
    }
}

// A tile of O(u) to the weights and their copies, or as it is.
template <bool Plan, int V>
__device__ __forceinline__ void finish_tile(const StreamArgs &a, const Place &p, const Matrix &q, const float (&x)[32]) {
    if constexpr (!Plan) {
        const size_t at = (size_t)p.matrix * p.g->rows * p.g->cols * 2;
        store_typed<V>(static_cast<unsigned char *>(a.y) + at, a.ytype, p.g->cols, p, x);
    } else {
        float w[32];
        load_tile<float, V>(w, q.w, p.g->cols, p);
#pragma unroll
        for (int k = 0; k < 32; ++k) w[k] = fmaf(-p.g->step, x[k], __fmul_rn(w[k], a.decay));
        store_tile<float, V>(q.w, p.g->cols, p, w);
        if (q.copy) store_typed<V>(q.copy, q.ctype, p.g->cols, p, w);
    }
}
template <bool Plan, int V>
__device__ __forceinline__ void last_tile(const StreamArgs &a, const Place &p, const Matrix &q) {
    float x[32];
    const __half *from = reinterpret_cast<const __half *>(a.tiles + (size_t)(p.g->x_last + p.matrix * p.g->per + p.tile) * kTileBytes);
    constexpr int kN = V;
#pragma unroll
    for (int k = 0; k < 32; k += kN) {
        const Run<__half, kN> r = *reinterpret_cast<const Run<__half, kN> *>(from + row_of<V>(k) * kTileCols + col_of<V>(k));
#pragma unroll
        for (int e = 0; e < kN; ++e) x[k + e] = __half2float(r.v[e]);
    }
    finish_tile<Plan, V>(a, p, q, x);
}
// A tile of A from its parts, in the first one's place; matrices `step` tiles apart.
__global__ void __launch_bounds__(kStreamThreads) k_gram_sum(unsigned char *tiles, const float *record, int base, int step, int gram_tiles,
                                                             int parts) {
    let_next_start();
    wait_for_previous();
    if (record && record[TULA_RECORD_FINITE] == 0.f) return;
    const int matrix = blockIdx.x / gram_tiles, tile = blockIdx.x - matrix * gram_tiles;
    unsigned char *const first = tiles + (size_t)(base + matrix * step + tile) * kTileBytes + threadIdx.x * 16;
#pragma unroll
    for (int at = 0; at < kTileBytes; at += kStreamThreads * 16) {
        float f[8] = {};
        for (int p = 0; p < parts; ++p) {
            const uint4 q = __ldcg(reinterpret_cast<const uint4 *>(first + (size_t)p * gram_tiles * kTileBytes + at));
            __half2 h[4];
            memcpy(h, &q, 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 v = __half22float2(h[k]);
                f[2 * k] += v.x;
                f[2 * k + 1] += v.y;
            }
        }
        __half2 h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2half2_rn(f[2 * k], f[2 * k + 1]);
        uint4 q;
        memcpy(&q, h, 16);
        *reinterpret_cast<uint4 *>(first + at) = q;
    }
}

template <bool Plan>
__global__ void __launch_bounds__(kStreamThreads, kStreamCtas<Plan>) k_muon_last(const __grid_constant__ StreamArgs a) {
    let_next_start();
    wait_for_previous();
    if (left_out(a)) return;
    const Place p = place_of(a, a.tile0 + blockIdx.x);
    Matrix q = {};
    if (Plan) q = a.matrices[p.g->matrix + p.matrix];
    switch (Plan ? q.vec : a.vec) {
        case 8: last_tile<Plan, 8>(a, p, q); break;
        case 2: last_tile<Plan, 2>(a, p, q); break;
        default: last_tile<Plan, 1>(a, p, q);
    }
}

// ----------------------------------------------------------------------------
// Small matrices
// ----------------------------------------------------------------------------
//
// One CTA a matrix whose smaller side is at most 128 and whose tiles, at most twelve, shared memory holds beside
// those of A, which B takes the place of.  Nothing leaves the SM between the first reading and the last
// writing: one launch and some 4 us a step instead of three launches and 13 (64 x 576: 38 us in all; 256 x 256 by
// the products above 74).  The tiles have the image that the copies give them there.  One thread issues a
// product, all eight warps read it back.

constexpr int kSmallTiles = 12;
constexpr int kSmallSmem = (kSmallTiles + 2) * kTileBytes + 1024;
constexpr int kSmallSums = 512;  // columns of sums at a time: all of tensor memory

// Where element (row, col) of a tile in shared memory lies, in bytes.
__device__ __forceinline__ uint32_t small_place(int row, int col) { return row * 128 + (((col >> 3) ^ (row & 7)) << 4) + (col & 7) * 2; }

struct Small {
    uint32_t x, gram, bar;
    volatile int *dead;
    uint32_t tmem;
    unsigned parity;

    // What the threads have written to shared memory, and read of tensor memory, comes before the next product.
    __device__ __forceinline__ void before() {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    // (a wait that runs out leaves the sums as they are: the others end at once then)
    __device__ __forceinline__ void after() {
        mbar_wait(bar, parity, dead);
        parity ^= 1;
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
};

template <bool Plan, int V>
__device__ __forceinline__ void small_load(const StreamArgs &a, Place p, const Matrix &q, int tiles, unsigned char *x, double *sums,
                                           float2 *factors) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = p.g->pitch;
    // (several tiles' parts are on their way at a time)
    constexpr int kAhead = Plan ? 2 : 4;
    auto tile = [&](int t) { p.row0 = t / pitch * kTile, p.col0 = t % pitch * kTileCols; };
    Loaded<Plan> l[kAhead];
    double total = 0.0;  // lane 0 of a warp
    for (int t0 = 0; t0 < tiles; t0 += kAhead) {
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            tile(t0 + h);
            if (t0 + h < tiles) load_parts<Plan, V>(l[h], a, p, q);
        }
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            if (t0 + h >= tiles) break;
            tile(t0 + h);
            float u[32];
            update_of<true, Plan, V>(u, l[h], a, p, q);
            warp_squares(u, sums);
            if (lane == 0) total += sums[warp];
        }
    }
    if (lane == 0) sums[warp] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int k = 0; k < kStreamThreads / 32; ++k) s += sums[k];
        *factors = factors_of(s, p.g->scale);
    }
    __syncthreads();
    const float2 f = *factors;
    constexpr int kN = V;
    for (int t0 = 0; t0 < tiles; t0 += kAhead) {
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            tile(t0 + h);
            if (t0 + h < tiles) load_parts<Plan, V>(l[h], a, p, q);
        }
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            if (t0 + h >= tiles) break;
            tile(t0 + h);
            float u[32];
            update_of<false, Plan, V>(u, l[h], a, p, q);
#pragma unroll
            for (int k = 0; k < 32; k += kN) {
                const Run<__half, kN> r = scaled_run<V>(u, k, p, f);
                *reinterpret_cast<Run<__half, kN> *>(x + (t0 + h) * kTileBytes + small_place(row_of<V>(k), col_of<V>(k))) = r;
            }
        }
    }
}
template <int V>
__device__ __forceinline__ void small_store(const StreamArgs &a, Place p, const Matrix &q, int tiles, const unsigned char *x) {
    const int pitch = p.g->pitch;
    for (int t = 0; t < tiles; ++t) {
        p.row0 = t / pitch * kTile, p.col0 = t % pitch * kTileCols;
        float f[32];
        constexpr int kN = V;
#pragma unroll
        for (int k = 0; k < 32; k += kN) {
            const Run<__half, kN> r =
                *reinterpret_cast<const Run<__half, kN> *>(x + t * kTileBytes + small_place(row_of<V>(k), col_of<V>(k)));
#pragma unroll
            for (int e = 0; e < kN; ++e) f[k + e] = __half2float(r.v[e]);
        }
        if (a.matrices)
            finish_tile<true, V>(a, p, q, f);
        else
            finish_tile<false, V>(a, p, q, f);
    }
}

// 64 columns of sums of a warp's 32 rows.
__device__ __forceinline__ void small_sums(float (&f)[64], uint32_t tmem) {
    unsigned v[64];
    tmem_load32(v, tmem);
    tmem_load32(v + 32, tmem + 32);
    tmem_wait(v);
#pragma unroll
    for (int k = 0; k < 64; ++k) f[k] = __uint_as_float(v[k]);
}
// A row of a tile, as fp16.
__device__ __forceinline__ void small_put(uint32_t tile, int row, const float (&f)[64]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        unsigned y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __half2 h = __floats2half2_rn(f[8 * k + 2 * e], f[8 * k + 2 * e + 1]);
            memcpy(&y[e], &h, 4);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tile + small_place(row, 8 * k)), "r"(y[0]), "r"(y[1]), "r"(y[2]),
                     "r"(y[3])
                     : "memory");
    }
}

__global__ void __launch_bounds__(kStreamThreads, 1) k_muon_small(const __grid_constant__ StreamArgs a, int steps) {
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ __align__(8) unsigned long long bar;
    __shared__ double sums[kStreamThreads / 32];
    __shared__ float2 factors;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    unsigned char *x = raw + (-smem_addr(raw) & 1023u);
    const int lane = threadIdx.x & 31, warp = __shfl_sync(kFull, threadIdx.x >> 5, 0);
    if (threadIdx.x == 0) {
        mbar_init(smem_addr(&bar), 1);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc(smem_addr(&tmem_at), kSmallSums);
    let_next_start();
    wait_for_previous();
    const Place p = place_of(a, blockIdx.x);  // (a group's tiles are its matrices here)
    const int rows = p.g->rows, cols = p.g->cols, n = min(rows, cols), pitch = p.g->pitch;
    const int tile_rows = (rows + kTile - 1) / kTile, tiles = tile_rows * pitch;
    const bool wide = rows <= cols, go = !left_out(a);
    Matrix q = {};
    if (a.matrices) q = a.matrices[p.g->matrix + p.matrix];
    const int vec = a.matrices ? q.vec : a.vec;
    Small m{smem_addr(x), smem_addr(x) + kSmallTiles * kTileBytes, smem_addr(&bar), &dead, 0, 0};
    if (go) {
        if (a.matrices) {
            switch (vec) {
                case 8: small_load<true, 8>(a, p, q, tiles, x, sums, &factors); break;
                case 2: small_load<true, 2>(a, p, q, tiles, x, sums, &factors); break;
                default: small_load<true, 1>(a, p, q, tiles, x, sums, &factors);
            }
        } else {
            switch (vec) {
                case 8: small_load<false, 8>(a, p, q, tiles, x, sums, &factors); break;
                case 2: small_load<false, 2>(a, p, q, tiles, x, sums, &factors); break;
                default: small_load<false, 1>(a, p, q, tiles, x, sums, &factors);
            }
        }
    }
    m.before();  // (and tensor memory is there)
    m.tmem = __shfl_sync(kFull, tmem_at, 0);
    const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane;
    const uint32_t lanes = m.tmem + ((unsigned)(quad * 32) << 16);
    const int sides = n > 64 ? 2 : 1;        // tiles to a row of A's
    const int parts = (n + 15) / 16;         // of a sum over the smaller side, an instruction each
    float scale = p.g->scale;
    for (int step = 0; go && step < steps; ++step) {
        // A = X X^T along X's tiles, or X^T X along their rows.  (There a tile beyond the last column may be read
        // as the rows beyond A's: they are not kept.)
        if (warp == 0) {
            if (elect_one()) {
                const uint32_t idesc = product_desc(128, 64 * sides, wide, wide);
                if (wide) {
                    for (int t = 0; t < pitch; ++t)
                        for (int j = 0; j < 4; ++j) {
                            const uint64_t d = operand_desc(m.x + t * kTileBytes, true) + 2 * j;
                            mma16<false>(m.tmem, d, d, idesc, t > 0 || j > 0);
                        }
                } else {
                    for (int t = 0; t < tile_rows; ++t)
                        for (int j = 0; j < 8; ++j) {
                            const uint64_t d = operand_desc(m.x + t * pitch * kTileBytes, false, kTileBytes) + 128 * j;
                            mma16<false>(m.tmem, d, d, idesc, t > 0 || j > 0);
                        }
                }
                commit(m.bar);
            }
            __syncwarp();
        }
        m.after();
        float f[64];
        if (half < sides) {
            const float alpha = 1.f / (scale * scale);
            small_sums(f, lanes + 64 * half);
#pragma unroll
            for (int k = 0; k < 64; ++k) f[k] = row < n && 64 * half + k < n ? f[k] * alpha : 0.f;
            small_put(m.gram + half * kTileBytes, row, f);
        }
        m.before();
        // B = a I + b A + c A^2, in A's place
        if (warp == 0) {
            if (elect_one()) {
                const uint32_t idesc = product_desc(128, 64 * sides, true, true);
                for (int j = 0; j < parts; ++j) {
                    const uint64_t d = operand_desc(m.gram + (j >> 2) * kTileBytes, true) + 2 * (j & 3);
                    mma16<false>(m.tmem, d, d, idesc, j > 0);
                }
                commit(m.bar);
            }
            __syncwarp();
        }
        m.after();
        if (half < sides) {
            small_sums(f, lanes + 64 * half);
            const int diagonal = row < n ? row - 64 * half : -1;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                unsigned y[4];
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3])
                             : "r"(m.gram + half * kTileBytes + small_place(row, 8 * k))
                             : "memory");
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    __half2 h;
                    memcpy(&h, &y[e >> 1], 4);
                    const float g = __half2float(e & 1 ? __high2half(h) : __low2half(h));
                    f[8 * k + e] = fmaf((float)kC, f[8 * k + e], fmaf((float)kB, g, diagonal == 8 * k + e ? (float)kA : 0.f));
                }
            }
            small_put(m.gram + half * kTileBytes, row, f);
        }
        // X' = B X by columns of tiles, or X B by rows of them, in X's place
        const int at_once = kSmallSums / 64;
        for (int t0 = 0; t0 < tiles; t0 += at_once) {
            const int t1 = min(tiles, t0 + at_once);
            m.before();
            if (warp == 0) {
                if (elect_one()) {
                    if (wide) {
                        for (int t = t0; t < t1; t += 4) {
                            const uint32_t idesc = product_desc(128, 64 * min(4, t1 - t), true, false);
                            for (int j = 0; j < parts; ++j)
                                mma16<false>(m.tmem + (t - t0) * 64, operand_desc(m.gram + (j >> 2) * kTileBytes, true) + 2 * (j & 3),
                                             operand_desc(m.x + t * kTileBytes, false, kTileBytes) + 128 * j, idesc, j > 0);
                        }
                    } else {
                        const uint32_t idesc = product_desc(128, 64 * sides, true, true);
                        for (int t = t0; t < t1; t += sides)
                            for (int j = 0; j < parts; ++j)
                                mma16<false>(m.tmem + (t - t0) * 64, operand_desc(m.x + (t + (j >> 2)) * kTileBytes, true) + 2 * (j & 3),
                                             operand_desc(m.gram + (j >> 2) * kTileBytes, true) + 2 * (j & 3), idesc, j > 0);
                    }
                    commit(m.bar);
                }
                __syncwarp();
            }
            m.after();
            const float alpha = 1.f / scale;
            for (int t = t0 + half; t < t1; t += 2) {
                small_sums(f, lanes + 64 * (t - t0));
#pragma unroll
                for (int k = 0; k < 64; ++k) f[k] *= alpha;
                small_put(m.x + t * kTileBytes, row, f);
            }
        }
        scale = 1.f;
        m.before();
    }
    if (go) {
        switch (vec) {
            case 8: small_store<8>(a, p, q, tiles, x); break;
            case 2: small_store<2>(a, p, q, tiles, x); break;
            default: small_store<1>(a, p, q, tiles, x);
        }
    }
    // No product may be under way when tensor memory is given back.  Where a wait has run out the others did not wait:
    // a millisecond is far more than they take.
    if (dead)
        for (int w = 0; w < 1000; ++w) __nanosleep(1000);
    __syncwarp();
    if (warp == 0) tmem_free(m.tmem, kSmallSums);
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

// Matrices of one shape.
struct Kin {
    long long rows, cols;
    int count, matrix;  // how many, the first one's place in the table
    int vec;            // as Matrix's
    float step;         // lr times the shape's factor
    int x0, x1, gram, poly;  // first tiles
    int tile_rows() const { return (int)up(rows, kTile); }
    int tile_cols() const { return (int)up(cols, kTileCols); }
    int tiles() const { return tile_rows() * tile_cols(); }
    bool fits() const { return std::min(rows, cols) <= 128 && up(rows, kTile) * up(cols, kTileCols) <= kSmallTiles; }
    bool wide() const { return rows <= cols; }
    long long n() const { return std::min(rows, cols); }
    int gram_rows() const { return (int)up(n(), kTile); }
    int gram_cols() const { return (int)up(n(), kTileCols); }
    int gram_tiles() const { return gram_rows() * gram_cols(); }
    // parts of A's sums, tiles of X from one to the next, and a part's stages
    int parts() const { return (int)up(std::max(rows, cols), kMostSum); }
    int part_step() const { return wide() ? kMostSum / kTileCols : kMostSum / kTile * tile_cols(); }
    int part_stages(int p) const { return (int)up(std::min<long long>(std::max(rows, cols) - (long long)p * kMostSum, kMostSum), 64); }
    // 2^s, s the whole part of log2(sqrt(rows cols)), at most 15: no element of X, 1 at most, leaves fp16's range
    int shift() const { return std::min(15, (int)std::floor(0.5 * std::log2((double)rows * (double)cols))); }
};

// Whether the list is k_muon_small's: where no matrix is larger (304 of 100 x 300 in 118 us, by products 225; 304 of
// 128 x 768 in 154, 374).  Else the products take the small ones along: 16 matrices of 17 to 700 rows and
// columns took 227 us by both, 160 by products alone.
bool all_small(const std::vector<Kin> &kin) {
    for (const Kin &k : kin)
        if (!k.fits()) return false;
    return true;
}

bool good_shape(long long rows, long long cols) { return rows >= 0 && cols >= 0 && rows <= kMostSide && cols <= kMostSide; }

// Gives every shape its tiles; returns how many there are, -1 beyond the limit.
long long place(std::vector<Kin> &kin) {
    long long at = 0;
    if (all_small(kin)) return 0;
    for (Kin &k : kin) {
        const long long x = (long long)k.tile_rows() * k.tile_cols() * k.count, a = (long long)k.gram_rows() * k.gram_cols() * k.count;
        const long long all = 2 * x + a * (k.parts() + 1);
        if (at + all >= kMostTiles) return -1;
        k.x0 = (int)at;
        k.x1 = (int)(at + x);
        k.gram = (int)(at + 2 * x);
        k.poly = (int)(at + 2 * x + a * k.parts());
        at += all;
    }
    return at;
}
long long stream_tiles(const Kin *kin, int n) {
    long long t = 0;
    for (int i = 0; i < n; ++i) t += (long long)kin[i].tiles() * kin[i].count;
    return t;
}

struct Maps {
    CUtensorMap in, out;
};
bool make_maps(Maps &m, const void *tiles, long long n) {
    const CUtensorMapDataType f16 = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return make_map(&m.in, f16, tiles, n * kTile, kTileCols, 128, 64, kTileCols, CU_TENSOR_MAP_SWIZZLE_128B) &&
           make_map(&m.out, f16, tiles, n * kTile, kTileCols, 128, 32, kTileCols, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool Pair, Kind K>
int launch_product(const Maps &maps, ProductArgs &a, int sms, cudaStream_t s) {
    using S = Shape<Pair>;
    static std::atomic<uint64_t> done;
    const int rc = allow_smem((const void *)k_product<Pair, K>, S::kSmem, &done);
    if (rc) return rc;
    const int workers = std::min(a.n_blocks, Pair ? std::max(1, sms / 2) : sms);
    int next = 1;  // the first group with other sums
    while (next < a.n_groups && a.g[next].n_k == a.g[0].n_k) ++next;
    a.n_first = next < a.n_groups ? a.g[next].first : a.n_blocks;
    a.skip = 0;
    const int more = a.n_first % workers, rest = a.n_blocks - a.n_first;
    if (more && rest > 0) {
        const int rounds = (a.g[0].n_k + a.g[next].n_k / 2) / a.g[next].n_k;
        a.skip = std::min(rounds, rest / (workers - more));  // whole rounds of those that are left
    }
    return tula::launch(k_product<Pair, K>, dim3((unsigned)(workers * (Pair ? 2 : 1))), kThreads, S::kSmem, s, Pair ? 2 : 1, maps.in,
                        maps.out, a);
}

// One product of all shapes (of A the sums' first part), or, part0 > 0, of one shape's A the parts from there on.  x:
// X's first tiles are x0 (0) or x1 (1); first: of the first step.
template <bool Pair>
int fill(ProductArgs &a, const Kin *kin, int n, Kind kind, int x, bool first, int part0) {
    constexpr int kSide = Shape<Pair>::kSide;
    long long blocks = 0;
    a.n_groups = part0 ? kin->parts() - part0 : n;
    for (int i = 0; i < a.n_groups; ++i) {
        const Kin &k = kin[part0 ? 0 : i];
        const int part = part0 ? part0 + i : 0;
        ProductGroup &g = a.g[i];
        const Side sx = {(x ? k.x1 : k.x0) + part * k.part_step(), k.tiles(), k.tile_cols(), k.tile_rows(), kAlong};
        const Side sa = {k.gram, k.gram_tiles() * k.parts(), k.gram_cols(), k.gram_rows(), kSymmetric};
        const Side sb = {k.poly, k.gram_tiles(), k.gram_cols(), k.gram_rows(), kSymmetric};
        Side across = sx;
        across.way = kAcross;
        g.n = (int)k.n();
        g.alpha = 1.f;
        g.finish = kind == kLast && k.vec == 8;
        g.rows = (int)k.rows;
        g.cols = (int)k.cols;
        g.matrix = k.matrix;
        g.step = k.step;
        if (kind >= kApply) {
            g.p = k.wide() ? sb : sx;
            g.q = k.wide() ? across : sb;
            g.out = x ? k.x0 : k.x1;
            g.out_step = k.tiles();
            g.out_pitch = k.tile_cols();
            g.out_rows = k.tile_rows();
            g.blocks_m = (int)up(k.rows, kSide);
            g.blocks_n = (int)up(k.cols, kSide);
            g.per = g.blocks_m * g.blocks_n;
            g.n_k = (int)up(k.n(), 64);
            if (first) g.alpha = (float)std::ldexp(1.0, -k.shift());
        } else {
            g.p = g.q = kind == kPoly ? sa : k.wide() ? sx : across;
            g.out = kind == kPoly ? k.poly : k.gram + part * k.gram_tiles();
            g.out_step = kind == kPoly ? k.gram_tiles() : k.gram_tiles() * k.parts();
            g.out_pitch = k.gram_cols();
            g.out_rows = k.gram_rows();
            g.blocks_m = g.blocks_n = (int)up(k.n(), kSide);
            long long per = 0;
            for (int c = 0; c < g.blocks_n; ++c) per += column_blocks<kSide>(c, g.blocks_n);
            if (per >= (1LL << 30)) return -1;
            g.per = (int)per;
            g.n_k = kind == kPoly ? (int)up(k.n(), 64) : k.part_stages(part);
            if (first && kind == kGram) g.alpha = (float)std::ldexp(1.0, -2 * k.shift());
        }
        g.first = (int)blocks;
        blocks += (long long)g.per * k.count;
        if (blocks >= (1LL << 30)) return -1;
    }
    a.n_blocks = (int)blocks;
    return (int)blocks;
}
template <Kind K>
int product(const Maps &maps, ProductArgs &a, const Kin *kin, int n, int x, bool first, int sms, cudaStream_t s, int part0 = 0) {
    const int pairs = fill<true>(a, kin, n, K, x, first, part0);
    const int singles = fill<false>(a, kin, n, K, x, first, part0);
    if (pairs < 0 || singles < 0) return TULA_ERR_ARG;
    // Blocks of 128 where each SM has one at most (1024 x 1024: 127 us, 153 by pairs); else pairs of CTAs where they need no more rounds, since a
    // round takes as long.
    if (singles > sms && up(pairs, std::max(1, sms / 2)) <= up(singles, sms)) {
        fill<true>(a, kin, n, K, x, first, part0);
        return launch_product<true, K>(maps, a, sms, s);
    }
    return launch_product<false, K>(maps, a, sms, s);
}
// A: its sums' first parts, those of long sides, and their sums.
int gram(const Maps &maps, ProductArgs &a, const Kin *kin, int n, int x, bool first, unsigned char *tiles, int sms, cudaStream_t s) {
    int rc = product<kGram>(maps, a, kin, n, x, first, sms, s);
    for (int i = 0; !rc && i < n; ++i) {
        const Kin &k = kin[i];
        if (k.parts() == 1) continue;
        rc = product<kGram>(maps, a, &k, 1, x, first, sms, s, 1);
        if (!rc)
            rc = tula::launch(k_gram_sum, dim3((unsigned)(k.gram_tiles() * k.count)), kStreamThreads, 0, s, 1, tiles, a.record, k.gram,
                              k.gram_tiles() * k.parts(), k.gram_tiles(), k.parts());
    }
    return rc;
}

// Small matrices, without a workspace.
int run_small(const Kin *kin, int n, StreamArgs &st, int steps, cudaStream_t s) {
    long long count = 0;
    st.n_groups = n;
    for (int i = 0; i < n; ++i) {
        const Kin &k = kin[i];
        Group &g = st.g[i];
        g = {};
        g.first = (int)count;
        g.per = 1;
        g.matrix = k.matrix;
        g.rows = (int)k.rows;
        g.cols = (int)k.cols;
        g.pitch = k.tile_cols();
        g.scale = steps ? (float)std::ldexp(1.0, k.shift()) : 1.f;
        g.step = k.step;
        count += k.count;
    }
    static std::atomic<uint64_t> done;
    const int rc = allow_smem((const void *)k_muon_small, kSmallSmem, &done);
    if (rc) return rc;
    return tula::launch(k_muon_small, dim3((unsigned)count), kStreamThreads, kSmallSmem, s, 1, st, steps);
}

// All of it for shapes whose tiles are placed (n_tiles 0: small ones), those with Kin::vec first.  `st`: its groups
// are filled here.
int run(const Maps &maps, long long n_tiles, const Kin *kin, int n, StreamArgs &st, int steps, cudaStream_t s) {
    if (!n_tiles) return n ? run_small(kin, n, st, steps, s) : TULA_OK;
    const int sms = std::max(1, sm_count());
    ProductArgs a;
    a.tiles = st.tiles;
    a.record = st.record;
    a.matrices = st.matrices;
    a.y = st.y;
    a.ytype = st.ytype;
    a.decay = st.decay;
    a.none = (int)(n_tiles * kTile);
    long long tiles = 0;
    st.n_groups = n;
    for (int i = 0; i < n; ++i) {
        const Kin &k = kin[i];
        Group &g = st.g[i];
        g.first = (int)tiles;
        g.per = k.tiles();
        g.matrix = k.matrix;
        g.rows = (int)k.rows;
        g.cols = (int)k.cols;
        g.pitch = k.tile_cols();
        g.x = k.x0;
        g.x_last = steps % 2 ? k.x1 : k.x0;
        g.scale = steps ? (float)std::ldexp(1.0, k.shift()) : 1.f;
        g.step = k.step;
        tiles += (long long)g.per * k.count;
    }
    if (tiles == 0) return TULA_OK;
    // (By parts of 48 MB, that the second of the two would find in L2, they take longer: 12 to 14 us a launch.)
    const bool plan = st.matrices != nullptr;
    int rc = tula::launch(plan ? k_muon_first<true> : k_muon_first<false>, dim3((unsigned)tiles), kStreamThreads, 0, s, 1, st);
    if (!rc) rc = tula::launch(plan ? k_muon_scale<true> : k_muon_scale<false>, dim3((unsigned)tiles), kStreamThreads, 0, s, 1, st);
    for (int i = 0; !rc && i < steps; ++i) {
        rc = gram(maps, a, kin, n, i & 1, i == 0, st.tiles, sms, s);
        if (!rc) rc = product<kPoly>(maps, a, kin, n, i & 1, i == 0, sms, s);
        if (!rc)
            rc = i == steps - 1 ? product<kLast>(maps, a, kin, n, i & 1, i == 0, sms, s)
                                : product<kApply>(maps, a, kin, n, i & 1, i == 0, sms, s);
    }
    // what the last product has not finished
    st.tile0 = 0;
    for (int i = 0; steps && i < n && kin[i].vec == 8; ++i) st.tile0 += st.g[i].per * kin[i].count;
    if (!rc && st.tile0 < tiles)
        rc = tula::launch(plan ? k_muon_last<true> : k_muon_last<false>, dim3((unsigned)(tiles - st.tile0)), kStreamThreads, 0, s, 1, st);
    return rc;
}

inline size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

struct tula_muon_plan {
    std::vector<Kin> kin;
    int dev;  // that it was made on
    Maps maps;
    long long n_tiles;
    const Matrix *matrices;
    double *parts;
    unsigned char *tiles;
};

namespace {

// The list's shapes, and which one each matrix is of (-1: empty).
bool shapes_of(const int64_t *rows, const int64_t *cols, const std::vector<int> *vec, int n, std::vector<Kin> &kin, std::vector<int> &which) {
    which.assign((size_t)n, -1);
    for (int i = 0; i < n; ++i) {
        if (!good_shape(rows[i], cols[i])) return false;
        if (rows[i] == 0 || cols[i] == 0) continue;
        const int v = vec ? (*vec)[(size_t)i] : 0;
        size_t k = 0;
        while (k < kin.size() && (kin[k].rows != rows[i] || kin[k].cols != cols[i] || kin[k].vec != v)) ++k;
        if (k == kin.size()) kin.push_back(Kin{rows[i], cols[i], 0, 0, v, 0.f, 0, 0, 0, 0});
        ++kin[k].count;
        which[i] = (int)k;
    }
    // those that the last product finishes first (see run), and the longest sums first, so that the last blocks to be
    // taken are short ones
    std::vector<int> order(kin.size()), where(kin.size());
    for (size_t k = 0; k < kin.size(); ++k) order[k] = (int)k;
    std::stable_sort(order.begin(), order.end(),
                     [&](int a, int b) {
                         if (kin[a].vec != kin[b].vec) return kin[a].vec > kin[b].vec;
                         return std::max(kin[a].rows, kin[a].cols) > std::max(kin[b].rows, kin[b].cols);
                     });
    std::vector<Kin> sorted;
    int first = 0;
    for (size_t k = 0; k < order.size(); ++k) {
        where[order[k]] = (int)k;
        sorted.push_back(kin[order[k]]);
        sorted.back().matrix = first;
        first += sorted.back().count;
    }
    for (int &w : which)
        if (w >= 0) w = where[w];
    kin.swap(sorted);
    return true;
}
// Whether a buffer that is written shares memory with another.  Gradients may with each other, and with their own
// matrix's weights or copy, which are written after the last reading of them.
bool overlapping(const std::vector<Matrix> &of, const int64_t *rows, const int64_t *cols) {
    struct Range {
        uintptr_t begin, end;
        bool written;
        bool holds(const Range &r) const { return begin <= r.begin && r.end <= end; }
    };
    std::vector<Range> all;
    for (size_t i = 0; i < of.size(); ++i) {
        const Matrix &q = of[i];
        if (!q.w) continue;
        auto range = [&](const void *p, int size, bool written) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p);
            return Range{at, at + (uintptr_t)rows[i] * (uintptr_t)cols[i] * (uintptr_t)size, written};
        };
        const Range g = range(q.g, type_size(q.gtype), false), w = range(q.w, 4, true), copy = range(q.copy, 2, true);
        all.push_back(w);
        all.push_back(range(q.m, 4, true));
        if (q.copy) all.push_back(copy);
        if (!w.holds(g) && !(q.copy && copy.holds(g))) all.push_back(g);
    }
    std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    uintptr_t end = 0, end_written = 0;  // of those before
    for (const Range &r : all) {
        if (r.begin < (r.written ? end : end_written)) return true;
        end = std::max(end, r.end);
        if (r.written) end_written = std::max(end_written, r.end);
    }
    return false;
}
struct Sizes {
    size_t table, parts, all;
    long long n_tiles;
};
bool sizes_of(std::vector<Kin> &kin, Sizes &z) {
    z.n_tiles = place(kin);
    if (z.n_tiles < 0) return false;
    size_t n = 0;
    for (const Kin &k : kin) n += (size_t)k.count;
    z.table = round_up(n * sizeof(Matrix));
    z.parts = z.n_tiles ? round_up((size_t)stream_tiles(kin.data(), (int)kin.size()) * sizeof(double)) : 0;
    z.all = z.table + z.parts + (size_t)z.n_tiles * kTileBytes;
    return true;
}

}  // namespace

extern "C" {

int tula_muon_workspace_size(const int64_t *rows, const int64_t *cols, int n_matrices, size_t *bytes) {
    if (!bytes || n_matrices < 0 || (n_matrices && (!rows || !cols))) return TULA_ERR_ARG;
    try {
        std::vector<Kin> kin;
        std::vector<int> which;
        Sizes z;
        if (!shapes_of(rows, cols, nullptr, n_matrices, kin, which) || !sizes_of(kin, z)) return TULA_ERR_ARG;
        *bytes = std::max<size_t>(z.all, 256);
    } catch (const std::bad_alloc &) {
        return TULA_ERR_NO_MEMORY;
    }
    return TULA_OK;
}

int tula_muon_plan_create(const tula_muon_matrices *m, void *workspace, size_t workspace_bytes, void *stream, tula_muon_plan **plan_out) {
    if (!plan_out) return TULA_ERR_ARG;
    *plan_out = nullptr;
    if (!m || m->n_matrices < 0) return TULA_ERR_ARG;
    const int n = m->n_matrices;
    if (n && (!m->rows || !m->cols || !m->grad_ptrs || !m->param_ptrs || !m->momentum_ptrs)) return TULA_ERR_ARG;
    try {
        std::unique_ptr<tula_muon_plan> plan(new tula_muon_plan);
        std::vector<int> which;
        Sizes z;
        std::vector<Matrix> of((size_t)n);
        std::vector<int> vec((size_t)n);
        for (int i = 0; i < n; ++i) {
            if (!good_shape(m->rows[i], m->cols[i])) return TULA_ERR_ARG;
            if (m->rows[i] == 0 || m->cols[i] == 0) continue;
            Matrix &q = of[(size_t)i];
            q = {};
            q.g = m->grad_ptrs[i];
            q.m = m->momentum_ptrs[i];
            q.w = m->param_ptrs[i];
            q.copy = m->copy_ptrs ? m->copy_ptrs[i] : nullptr;
            q.gtype = m->grad_types ? m->grad_types[i] : TULA_TYPE_F32;
            q.ctype = m->copy_types ? m->copy_types[i] : TULA_TYPE_BF16;
            if (!good_type(q.gtype) || (q.ctype != TULA_TYPE_BF16 && q.ctype != TULA_TYPE_F16) || !q.g || !q.m || !q.w ||
                (m->copy_ptrs && !q.copy) || !aligned(q.g, type_size(q.gtype)) || !aligned(q.m, 4) || !aligned(q.w, 4) ||
                !aligned(q.copy, 2))
                return TULA_ERR_ARG;
            const unsigned two = 2 * type_size(q.gtype);
            if (m->cols[i] % 8 == 0 && aligned(q.g, 16) && aligned(q.m, 16) && aligned(q.w, 32) && aligned(q.copy, 16))
                q.vec = 8;
            else
                q.vec = m->cols[i] % 2 == 0 && aligned(q.g, two) && aligned(q.m, 8) && aligned(q.w, 8) && aligned(q.copy, 4) ? 2 : 1;
            vec[(size_t)i] = q.vec;
        }
        if (!shapes_of(m->rows, m->cols, &vec, n, plan->kin, which) || !sizes_of(plan->kin, z)) return TULA_ERR_ARG;
        std::vector<int> next(plan->kin.size(), 0);
        std::vector<Matrix> table(z.table / sizeof(Matrix));
        for (int i = 0; i < n; ++i)
            if (which[i] >= 0) table[(size_t)(plan->kin[which[i]].matrix + next[which[i]]++)] = of[(size_t)i];
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < std::max<size_t>(z.all, 256)) return TULA_ERR_WORKSPACE;
        if (overlapping(of, m->rows, m->cols)) return TULA_ERR_ARG;
        unsigned char *at = static_cast<unsigned char *>(workspace);
        plan->n_tiles = z.n_tiles;
        plan->matrices = reinterpret_cast<const Matrix *>(at);
        plan->parts = reinterpret_cast<double *>(at + z.table);
        plan->tiles = at + z.table + z.parts;
        std::memset(&plan->maps, 0, sizeof(plan->maps));
        if (z.table) {
            cudaStream_t s = static_cast<cudaStream_t>(stream);
            cudaError_t e = cudaGetDevice(&plan->dev);
            if (e == cudaSuccess) e = cudaMemcpyAsync(at, table.data(), table.size() * sizeof(Matrix), cudaMemcpyHostToDevice, s);
            if (e == cudaSuccess) e = cudaStreamSynchronize(s);
            if (e != cudaSuccess) return cuda_failed(e);
            if (z.n_tiles && !make_maps(plan->maps, plan->tiles, z.n_tiles)) return cuda_failed(cudaErrorInvalidValue);
        }
        *plan_out = plan.release();
    } catch (const std::bad_alloc &) {
        return TULA_ERR_NO_MEMORY;
    }
    return TULA_OK;
}

int tula_muon_plan_destroy(tula_muon_plan *plan) {
    delete plan;
    return TULA_OK;
}

void tula_muon_default_hparams(tula_muon_hparams *hp) {
    if (!hp) return;
    *hp = tula_muon_hparams{};
    hp->lr = 1e-3;
    hp->momentum = 0.95;
    hp->grad_scale = 1.0;
    hp->nesterov = 1;
    hp->ns_steps = 5;
    hp->scale = TULA_MUON_SCALE_RMS;
}

int tula_muon_step(tula_muon_plan *plan, const tula_muon_hparams *hp, void *stream) {
    if (!plan || !hp) return TULA_ERR_ARG;
    const bool good = hp->lr >= 0 && hp->lr <= 1e30 && hp->momentum >= 0 && hp->momentum < 1 && hp->weight_decay >= 0 &&
                      hp->weight_decay <= 1e30 && hp->grad_scale >= 0x1p-100 && hp->grad_scale <= 0x1p100 && hp->ns_steps >= 0 &&
                      hp->ns_steps <= kMostSteps && (hp->scale == TULA_MUON_SCALE_RMS || hp->scale == TULA_MUON_SCALE_ASPECT) &&
                      aligned(hp->record, 4);
    if (!good) return TULA_ERR_ARG;
    const int n = (int)plan->kin.size();
    if (!n) return TULA_OK;
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_failed(e);
    if (dev != plan->dev) return TULA_ERR_ARG;
    StreamArgs st = {};
    st.matrices = plan->matrices;
    st.tiles = plan->tiles;
    st.record = hp->record;
    st.grad_scale = (float)hp->grad_scale;
    st.mu = (float)hp->momentum;
    st.decay = (float)(1.0 - hp->lr * hp->weight_decay);
    st.nesterov = hp->nesterov != 0;
    long long done = 0;
    for (int i = 0; i < n; i += kMostGroups) {
        const int here = std::min(kMostGroups, n - i);
        Kin kin[kMostGroups];
        for (int k = 0; k < here; ++k) {
            kin[k] = plan->kin[(size_t)(i + k)];
            const double r = (double)kin[k].rows, c = (double)kin[k].cols;
            const double factor = hp->scale == TULA_MUON_SCALE_RMS ? 0.2 * std::sqrt(std::max(r, c)) : std::sqrt(std::max(1.0, r / c));
            kin[k].step = (float)(hp->lr * factor);
        }
        st.parts = plan->parts + done;
        done += stream_tiles(kin, here);
        const int rc = run(plan->maps, plan->n_tiles, kin, here, st, hp->ns_steps, static_cast<cudaStream_t>(stream));
        if (rc) return rc;
    }
    return TULA_OK;
}

int tula_orthogonalize_workspace_size(int64_t batch, int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes || batch < 0 || !good_shape(rows, cols) || batch >= kMostTiles) return TULA_ERR_ARG;
    *bytes = 256;
    if (batch == 0 || rows == 0 || cols == 0) return TULA_OK;
    try {
        std::vector<Kin> kin{Kin{rows, cols, (int)batch, 0, 0, 0.f, 0, 0, 0, 0}};
        Sizes z;
        if (!sizes_of(kin, z)) return TULA_ERR_ARG;
        *bytes = std::max<size_t>(z.parts + (size_t)z.n_tiles * kTileBytes, 256);
    } catch (const std::bad_alloc &) {
        return TULA_ERR_NO_MEMORY;
    }
    return TULA_OK;
}

int tula_orthogonalize(const void *x, int type, int64_t batch, int64_t rows, int64_t cols, int64_t stride, int64_t batch_stride, int ns_steps,
                       void *out, int out_type, void *workspace, size_t workspace_bytes, void *stream) {
    size_t need = 0;
    const int rc = tula_orthogonalize_workspace_size(batch, rows, cols, &need);
    if (rc) return rc;
    if (!good_type(type) || (out_type != TULA_TYPE_BF16 && out_type != TULA_TYPE_F16) || stride < cols || batch_stride < 0 || ns_steps < 0 ||
        ns_steps > kMostSteps)
        return TULA_ERR_ARG;
    if (batch == 0 || rows == 0 || cols == 0) return TULA_OK;
    if (!x || !out || !aligned(x, type_size(type)) || !aligned(out, 2)) return TULA_ERR_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return TULA_ERR_WORKSPACE;
    try {
        std::vector<Kin> kin{Kin{rows, cols, (int)batch, 0, 0, 0.f, 0, 0, 0, 0}};
        Sizes z;
        if (!sizes_of(kin, z)) return TULA_ERR_ARG;
        StreamArgs st = {};
        st.x = x;
        st.xtype = type;
        st.stride = stride;
        st.batch_stride = batch_stride;
        st.y = out;
        st.ytype = out_type;
        st.parts = static_cast<double *>(workspace);
        st.tiles = static_cast<unsigned char *>(workspace) + z.parts;
        st.grad_scale = 1.f;
        const size_t size = type_size(type);
        auto lies = [&](unsigned n, unsigned bytes) {  // runs of n elements at boundaries of n, or of so many bytes
            const unsigned at = std::min<unsigned>(n, 16 / (unsigned)size);
            return cols % n == 0 && aligned(x, at * (unsigned)size) && aligned(out, bytes) && (rows == 1 || stride % at == 0) &&
                   (batch == 1 || batch_stride % at == 0);
        };
        st.vec = lies(8, 16) ? 8 : lies(2, 4) ? 2 : 1;
        kin[0].vec = st.vec;
        Maps maps;
        std::memset(&maps, 0, sizeof(maps));
        if (z.n_tiles && !make_maps(maps, st.tiles, z.n_tiles)) return cuda_failed(cudaErrorInvalidValue);
        return run(maps, z.n_tiles, kin.data(), 1, st, ns_steps, static_cast<cudaStream_t>(stream));
    } catch (const std::bad_alloc &) {
        return TULA_ERR_NO_MEMORY;
    }
}

int tula_muon_check_wait_timeout(void *stream) { return check_wait_timeout(stream); }

int tula_muon_error(void *stream, int *error_out) { return read_error(stream, error_out); }

}  // extern "C"
