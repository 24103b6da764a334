// Newton-Schulz orthogonalisation of a batch of matrices:  X = G / (|G|_F + eps);  steps times  A = X X^T,  X <- a X + (b A + c A A) X.
// With X = U S V^T a step takes every singular value x to a x + b x^3 + c x^5 and leaves U and V alone.  The short side is the rows
// of X (a tall G is read and written transposed), so that A is s x s; it and its polynomial are symmetric and half their tiles are made.
// Bound by the matrix instructions where there are many tiles, by launches and latencies where there are few.  (A short side of at most 128:
// r3_ortho_narrow.hip.)
//
// Numbers.  The matrix instruction's f16 operands, f32 sums.  A step's values are known beforehand: |X|_2 stays below about 1.2, so no
// element of X, A or B = b A + c A A leaves (-16, 16) (the host checks it for other coefficients), and everything is stored times 2^12: at
// best 11 bits, four times bf16's, down to 1.5e-8.  A rounding of X is an error that the coming steps multiply by up to a each (a small
// singular value grows by a, a new one beside it does too), so while three steps and more are left X is kept as an f16 and 8 bits of what
// its rounding leaves; the f16 alone enters the products, where the small directions hardly count.  The last two steps' polynomial has a +
// b + c, what it is for singular values of 1, taken out of B and applied to X in f32, so that B's rounding is one of a small matrix.
// Relative error of bf16 results in the Frobenius norm, beside their own rounding (1.7e-3), at 256 x 768 and 768 x 2048: 7e-4 ... 1.1e-3 for
// matrices with flat and falling spectra; 4e-3, 5e-3, 4e-3, 7.5e-3 for those of four, three, two and one directions, where what X's 8 bits leave
// grows by a in every other direction (simulated with 11 bits: 3e-3; in the 2-norm, rounding included, all four are 9e-4 ... 1.8e-3); with bf16
// operands throughout it is 1e-2 ... 4e-2.  For f32 results all of X, A, B are pairs of f16 and products are the three of their parts that count
// (hi lo, lo hi, hi hi): 22 bits, 1.3e-6 ... 3e-6 and, of few directions, 2.4e-5 ... 8.2e-5, where the same steps in f32 on a CPU have 1.6e-6 ...
// 2.4e-5 and 2.5e-5 ... 1.2e-4.
//
// 128 of 2048 x 768 f32 to bf16 3550 us, 32 of 768 x 2048 to f32 2132; the products alone would be 1992 and (three to one) 1493 at the 1.31
// PFLOP/s of a large f16 product.  X X^T runs at 1.08 PFLOP/s (190 us), the products with X at 0.70 ... 0.85 (441 with X's 8 bits, 364
// without): their results, as large as X, are written when a tile is done and no second work-group fits beside it to multiply meanwhile.
// (Tiles of 128 x 256 with two to a compute unit took as long, bound by the L2; fewer matrices at a time, so that X stays in the caches,
// longer.)
#include <algorithm>
#include <cmath>
#include <utility>

#include "r3_kernels.h"
#include "r3_mfma2.h"
#include "r3_vec.h"

namespace r3 {
namespace {

typedef _Float16 f16_t;
typedef f16_t f16x4_t __attribute__((ext_vector_type(4)));

constexpr int kSide = 128;                 // of a block of results; a work-group has two by two
constexpr float kUnit = 4096.0f;           // what is stored is times this
constexpr int kPitchF = kSide + 4;         // of a tile of results in LDS
constexpr int kLdsTile = kSide * kPitchF * 4;   // 66 KB: 128 x 128 results; two of them, where the windows or stages of operands were
static_assert(2 * kLdsTile >= 2 * kSuperBytes && 2 * kLdsTile >= kStages2 * kStageBytes, "");

struct Pair { f16_t *hi, *lo; };   // (lo: f16, or X's 8 bits where only hi is multiplied)

// A launch's product D[q][p] = sum_k Q[q][k] P[p][k] per matrix and what is made of it, all in units of 1 / kUnit:
//   result = cd (D + own P) + c1 E1 + c2 E2 + diag I
// kSquare: q, p < s, symmetric, lower half and its mirror image; kStep: p < l; kStepLow: the same with c1 times the 8 bits of E1 (if there
// are any) and 8 bits of its own (if dst has a place for them); kLast: as kStep, times `out`, to the caller's array.
// own P costs no loads: where a tile's k are its own rows the operand is in LDS, and is multiplied with `own` times a unit matrix, too
// (two f16, so that `own` keeps 22 bits).
enum { kGram = 0, kSquare = 1, kStep = 2, kStepLow = 3, kLast = 4 };
struct Product {
    int s, l, sp, lp;              // X is s x l in sp x lp, A and the like s x s in sp x sp, zeros beyond
    int ntiles;                    // of a matrix
    int passes;                    // through k: 1, or 3 for pairs (as a constant of the loop it costs registers that spill)
    Pair Q, P, E1, E2, dst;        // (E1: or none; E2: or none, large tiles alone)
    f16_t own, own_lo;             // times kUnit
    float cd, c1, c2, diag, out;
    void *O;
    bool transposed;
};
// `own` times columns 16 j .. + 15 of a unit matrix of 32 rows, as an operand's fragment
__device__ __forceinline__ bf16x8_t unit_part(int lane, int j, f16_t own) {
    const int at = 16 * j + (lane & 15) - 8 * (lane >> 4);
    f16x8_t v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at == e ? own : (f16_t)0.0f;
    return __builtin_bit_cast(bf16x8_t, v);
}

// All but LOADS of this wave's loads have landed and everybody has left the stage before, whose place the next loads take.
template <int LOADS = 0> __device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    window_barrier<LOADS>();
    asm volatile("" ::: "memory");
}

// `PARTS` of the operations below: 1: hi hi; 3: lo hi, hi lo, hi hi, one pass through k after the other (`low`: which takes an operand's lo)

// Operands with k along their rows (X in X X^T) for the tile loop of r3_mfma2.h: windows of 64 k of 256 rows, a pass behind the other.
// Rows past the last matrix's last read zeros, those past another's are the next one's, in results that nobody stores.
template <int PARTS> struct RowsOp {
    static constexpr bool kIndexed = false, kWindowed = true;
    static constexpr int kReads = 1;
    typedef MfmaF16 Mfma;
    rsrc_t hi, lo;
    int nw, low, voff, step;
    KcFrag16 fr;
    // `bytes`: from the tile's first row to the end of all matrices
    __device__ __forceinline__ void init(const f16_t *h, const f16_t *l, uint64_t bytes, int ld, int nw_, int low_, int wave_base) {
        hi = src_rsrc(Src{(const char *)h, bytes, 0u}, 0);
        if constexpr (PARTS == 3) lo = src_rsrc(Src{(const char *)l, bytes, 0u}, 0);
        nw = nw_;
        low = low_;
        const int w = threadIdx.x >> 6, lane = lane_id(), row = 8 * (w & 3) + (lane >> 3);
        voff = row * ld + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        step = __builtin_amdgcn_readfirstlane(32 * ld);
        fr.init(wave_base, lane);
    }
    __device__ __forceinline__ void issue_window(int J, uint32_t win, int = kTile) const {
        const int pass = PARTS == 3 ? (J >= nw) + (J >= 2 * nw) : 0;
        const rsrc_t r = PARTS == 3 && pass == low ? lo : hi;
        const int adv = (J - pass * nw) * (kBK3 * 2), w = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int sum = adv + i * step;
            asm("" : "+s"(sum));
            lds_load16(r, win + 1024 * ((w & 3) + kLoaderWaves * i), voff + sum);
        }
    }
    __device__ __forceinline__ bf16x8_t frag_window(const char *win, int t, int u) const { return fr.read(win, t, u); }
};

// Operands whose k-rows are rows in memory (X, and symmetric matrices, whose rows and columns are the same): stages of 32 k of 256
// columns.  Columns past a row's end are the next row's, in results that nobody stores; past the last matrix they are zeros.
struct ColumnsOp {
    const char *hi, *lo;
    uint64_t bytes;
    uint32_t step;
    int nk, low;     // (low < 0: hi alone)
    DmaTR<256> dma;
    TrFrag16<256> fr;
    // `bytes`: from the tile's first element to the end of all matrices
    __device__ __forceinline__ void init(const f16_t *h, const f16_t *l, uint64_t bytes_, int ld, int nk_, int low_, int wave_base) {
        hi = (const char *)h;
        lo = (const char *)l;
        bytes = bytes_;
        step = 32u * ld;
        nk = nk_;
        low = low_;
        dma.init(ld, 0);
        fr.init(wave_base);
    }
    __device__ __forceinline__ void issue(int kt, uint32_t tile) const {
        const int pass = (kt >= nk) + (kt >= 2 * nk);
        dma.issue(src_rsrc(Src{pass == low ? lo : hi, bytes, step}, kt - pass * nk), tile);
    }
};

// 256 x 256 in the ring of stages of r3_mfma2.h (its sub-steps, its waves' shares).  Where a stage's k are a wave's own rows, 64 of them in
// two stages from own_at, P meets `own` times a unit matrix, too (P's lo in its own pass).
__device__ __forceinline__ void multiply_columns(Acc2 &acc, int passes, const ColumnsOp &P, const ColumnsOp &Q, int own_at, f16_t own, f16_t own_lo,
                                                 char *lds) {
    const uint32_t at = lds_addr(lds);
    const bool loader = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) < kLoaderWaves;
    const int nk = P.nk, n = passes * nk;
    auto issue = [&](int kt) {
        const uint32_t to = at + (kt & 3) * kStageBytes;
        P.issue(kt, to);
        Q.issue(kt, to + kOperandBytes);
    };
    if (loader) issue(0);
    if (loader && n > 1) issue(1);
    if (n > 1) stage_barrier<8>(loader);
    else stage_barrier<0>(loader);
    Frags f;
    f.clear();
    int own_in = own_at, now = 0;     // stages until this wave's own rows; the pass
#pragma nounroll
    for (int kt = 0; kt < n; ++kt) {
        const char *st = lds + (kt & 3) * kStageBytes;
        auto fp = [&](int i) { return P.fr.read(st, i); };
        auto fq = [&](int j) { return Q.fr.read(st + kOperandBytes, j); };
        ring_first<MfmaF16>(acc, f, fp, fq);
        if (loader && kt + 2 < n) issue(kt + 2);
        __builtin_amdgcn_sched_barrier(0);
        ring_second<MfmaF16>(acc, f, fp, fq);
#pragma unroll
        for (int z = 0; z < 2; ++z)
            if (own_in == -z && now != 1) {
                int lane = lane_id();
                asm volatile("" : "+v"(lane));     // (made here, or the fragments are kept in registers all the way)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8_t e = unit_part(lane, j, own), el = unit_part(lane, j, own_lo);
#pragma unroll
                    for (int i = 0; i < kTP2; ++i) {
                        const bf16x8_t &p = i < kHalfP ? f.y[i % kHalfP] : f.x[i % kHalfP];
                        acc[i][2 * z + j] = MfmaF16::run(p, el, acc[i][2 * z + j]);
                        acc[i][2 * z + j] = MfmaF16::run(p, e, acc[i][2 * z + j]);
                    }
                }
            }
        if (own_at - own_in == nk - 1) {
            own_in = own_at;
            ++now;
        } else --own_in;
        if (kt + 2 < n) stage_barrier<8>(loader);
        else stage_barrier<0>(loader);
    }
    step_last<MfmaF16>(acc, f);
}

__device__ __forceinline__ f16_t part_hi(float v) { return (f16_t)v; }
__device__ __forceinline__ f16_t part_lo(float v, f16_t hi) { return (f16_t)(v - (float)hi); }

// A tile of results in LDS, row q at q (N + 4) with its columns' fours exchanged by q / 8, so that eight rows' values of a column, 16 x 4
// of them to a wave, meet at most two at a time in a bank; col is a multiple of 8 (read_down: row).
template <int N> __device__ __forceinline__ int sums_at(int q, int p) { return q * (N + 4) + (p ^ (((q >> 3) & 7) << 2)); }
template <int N> __device__ __forceinline__ void read_along(const float *sums, int row, int col, float *v) {
    *(f32x4_t *)v = *(const f32x4_t *)(sums + sums_at<N>(row, col));
    *(f32x4_t *)(v + 4) = *(const f32x4_t *)(sums + sums_at<N>(row, col + 4));
}
template <int N> __device__ __forceinline__ void read_down(const float *sums, int row, int col, float *v) {
    const float *at = sums + sums_at<N>(row, col);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = at[u * (N + 4)];
}
// What an f16 leaves of a value where it is not multiplied (X's, bf16 results): 8 bits with 2 of mantissa, times 2^8, which takes 1e-3 to 2^4
// times kUnit's results to the middle of their range.  A quarter less to move than with f16 (128 of 2048 x 768: the start 300 -> 257 us), for
// less exactness in matrices of few directions (above).
constexpr float kLow = 256.0f;
__device__ __forceinline__ uint2 pack_low(const float *v, const f16x8_t &h) {
    float r[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) r[u] = (v[u] - (float)h[u]) * kLow;
    int a = __builtin_amdgcn_cvt_pk_bf8_f32(r[0], r[1], 0, false), b = __builtin_amdgcn_cvt_pk_bf8_f32(r[4], r[5], 0, false);
    a = __builtin_amdgcn_cvt_pk_bf8_f32(r[2], r[3], a, true);
    b = __builtin_amdgcn_cvt_pk_bf8_f32(r[6], r[7], b, true);
    return make_uint2((unsigned)a, (unsigned)b);
}
__device__ __forceinline__ void add_low(const uint2 &low, float c, float *v) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const f32x2_t r[4] = {__builtin_amdgcn_cvt_pk_f32_bf8((int)low.x, false), __builtin_amdgcn_cvt_pk_f32_bf8((int)low.x, true),
                          __builtin_amdgcn_cvt_pk_f32_bf8((int)low.y, false), __builtin_amdgcn_cvt_pk_f32_bf8((int)low.y, true)};
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = fmaf(c * (1.0f / kLow), r[u >> 1][u & 1], v[u]);
}
// eight values to their place, and what their rounding leaves: nothing of it, an f16 or 8 bits
enum { kNoRest = 0, kRest16 = 1, kRest8 = 2 };
template <int REST> __device__ __forceinline__ void put8(const Pair &dst, int64_t e, const float *v) {
    f16x8_t h, lo;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        h[u] = part_hi(v[u]);
        lo[u] = part_lo(v[u], h[u]);
    }
    *(f16x8_t *)(dst.hi + e) = h;
    if constexpr (REST == kRest16) *(f16x8_t *)(dst.lo + e) = lo;
    if constexpr (REST == kRest8) *(uint2 *)((char *)dst.lo + e) = pack_low(v, h);
}
// v += c times eight values
template <bool LO> __device__ __forceinline__ void add8(const Pair &src, int64_t e, float c, float *v) {
    const f16x8_t h = *(const f16x8_t *)(src.hi + e);
    f16x8_t lo;
    if constexpr (LO) lo = *(const f16x8_t *)(src.lo + e);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = fmaf(c, LO ? (float)h[u] + (float)lo[u] : (float)h[u], v[u]);
}

// where tile (ti, tj) of a result begins, and the distance of its rows
template <int MODE, int N> __device__ __forceinline__ int64_t tile_at(const Product &o, int64_t m, int ti, int tj, int64_t &ld) {
    constexpr bool kSq = MODE == kGram || MODE == kSquare;
    ld = kSq ? o.sp : o.lp;
    return m * o.sp * ld + (int64_t)ti * N * ld + (int64_t)tj * N;
}
// What is made of an N x N tile of sums, rows of block ti and columns of block tj, by 256 threads.  Through LDS, so that whole lines are read
// and written; everybody meets between the two.
template <int MODE, bool SPLIT, int N, typename OUT>
__device__ __forceinline__ void finish_rows(const Product &o, int64_t m, int ti, int tj, float *sums, int tid) {
    constexpr bool kMirror = MODE == kGram || MODE == kSquare;
    int64_t ld;
    const int64_t tile = tile_at<MODE, N>(o, m, ti, tj, ld);
    const bool mirror = kMirror && ti != tj;
    // Eight columns of a row to a thread at a time.  X's lo: some loads together, one behind the other's stores their latencies were most
    // of the time.
    constexpr bool kAddLow = MODE == kStepLow;
    constexpr int kEach = N * N / 8 / 256, kBatch = kAddLow ? (kEach < 4 ? kEach : 4) : 1;
    for (int k0 = 0; k0 < kEach; k0 += kBatch) {
        uint2 low[kBatch];
        if (kAddLow && o.E1.lo) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int c = tid + 256 * (k0 + k);
                low[k] = *(const uint2 *)((const char *)o.E1.lo + tile + (int64_t)(c / (N / 8)) * ld + c % (N / 8) * 8);
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int c = tid + 256 * (k0 + k), r = c / (N / 8), col = c % (N / 8) * 8;
            const int64_t e = tile + (int64_t)r * ld + col;
            float v[8];
            read_along<N>(sums, r, col, v);
            if constexpr (MODE == kSquare) {
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] *= o.cd;
                if (o.E1.hi) add8<SPLIT>(o.E1, e, o.c1, v);
                const int row = ti * N + r;
                if (ti == tj && row < o.s) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) v[u] += row == tj * N + col + u ? o.diag : 0.0f;
                }
            }
            if (kAddLow && o.E1.lo) add_low(low[k], o.c1, v);
            if constexpr (MODE == kLast) {
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] *= o.out;
            }
            if (MODE == kLast || (MODE == kSquare && mirror)) {
#pragma unroll
                for (int u = 0; u < 8; u += 4) *(f32x4_t *)(sums + sums_at<N>(r, col + u)) = *(const f32x4_t *)(v + u);
            }
            if constexpr (MODE == kStepLow) {
                if (o.dst.lo) put8<kRest8>(o.dst, e, v);
                else put8<kNoRest>(o.dst, e, v);
            } else if constexpr (MODE != kLast) put8<SPLIT ? kRest16 : kNoRest>(o.dst, e, v);
        }
    }
}
template <int MODE, bool SPLIT, int N, typename OUT>
__device__ __forceinline__ void finish_rest(const Product &o, int64_t m, int ti, int tj, const float *sums, int tid) {
    if constexpr (MODE == kLast) {
        const int rows = o.transposed ? o.l : o.s, cols = o.transposed ? o.s : o.l;
        const int r0 = (o.transposed ? tj : ti) * N, c0 = (o.transposed ? ti : tj) * N;
        OUT *out = (OUT *)o.O + m * rows * cols;
        for (int k = 0; k < N * N / 8 / 256; ++k) {
            const int e = tid + 256 * k, r = e / (N / 8), c = e % (N / 8) * 8;
            if (r0 + r >= rows || c0 + c >= cols) continue;
            float v[8];
            if (o.transposed) read_down<N>(sums, c, r, v);
            else read_along<N>(sums, r, c, v);
            OUT *at = out + (int64_t)(r0 + r) * cols + c0 + c;
            if (c0 + c + 8 <= cols) {
#pragma unroll
                for (int u = 0; u < 8; u += Row<OUT>::kVec) Row<OUT>::store(at + u, v + u);
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (c0 + c + u < cols) Elem<OUT>::st(at + u, v[u]);
            }
        }
    }
    if constexpr (MODE == kGram || MODE == kSquare) {
        if (ti == tj) return;
        // the mirror image: eight rows' values of one column to a thread
        int64_t ld;
        const int64_t mirrored = tile_at<MODE, N>(o, m, tj, ti, ld);
#pragma unroll 2
        for (int k = 0; k < N * N / 8 / 256; ++k) {
            const int c = tid + 256 * k, r = c / (N / 8), col = c % (N / 8) * 8;
            float v[8];
            read_down<N>(sums, col, r, v);
            put8<SPLIT ? kRest16 : kNoRest>(o.dst, mirrored + (int64_t)r * ld + col, v);
        }
    }
}

// where a work-group's number takes it: the groups of an XCD (every eighth) have neighbouring tiles, and so the same matrices in its L2
__device__ __forceinline__ int64_t xcd_share(int64_t id, int64_t n) {
    const int64_t x = id & 7, q = n >> 3, r = n & 7;
    return x * q + (x < r ? x : r) + (id >> 3);
}

// A lane's sums of a block of NI x NJ 16 x 16: rows q0 + 16 j + (lane & 15), columns p0 + 16 i + 4 (lane >> 4) .. + 3.
template <int N, int NI, int NJ>
__device__ __forceinline__ void put_sums(const f32x4_t (&acc)[NI][NJ], int p0, int q0, float *sums) {
    const int lane = lane_id();
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)   // (both operands are times kUnit)
            *(f32x4_t *)(sums + sums_at<N>(q0 + 16 * j + (lane & 15), p0 + 16 * i + 4 * (lane >> 4))) = acc[i][j] * (1.0f / kUnit);
}

// ---- the ends of 256 x 256 tiles ----
// Where a result needs nothing but its sums it is rounded in registers, and the whole tile is f16 in
// LDS, where the operands were (pairs: hi, then lo): one round trip, and whole lines to memory.  (With f32 sums in LDS, two blocks of 128 x
// 128 at a time (below): 128 products of 768 x 768 117 us instead of 112, their last products with X of 768 x 2048, to bf16 443 instead of
// 419.)
constexpr int kPitch16 = kTile + 8;
static_assert(kTile * kPitch16 * 2 <= 2 * kLdsTile, "");

template <int MODE, bool SPLIT>
__device__ __forceinline__ void finish_rounded(const Product &o, int64_t m, int ti, int tj, int blocks, const Acc2 &acc, char *lds) {
    constexpr bool kSq = MODE == kGram || MODE == kSquare;
    f16_t *t = (f16_t *)lds;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), pw = wave & 1, qw = wave >> 1;
    const int r = lane & 15, c = 4 * (lane >> 4);
    int64_t ld;
    const int64_t tile = tile_at<MODE, kTile>(o, m, ti, tj, ld);
    const float unit = MODE == kSquare ? o.cd * (1.0f / kUnit) : 1.0f / kUnit;   // (both operands are times kUnit)
    // (blocks of 128 x 128: h down, g along)
    auto wanted = [&](int h, int g) { return 2 * ti + h < o.sp / kSide && 2 * tj + g < blocks && (!kSq || 2 * tj + g <= 2 * ti + h); };
    const bool mine = wanted(qw >> 1, pw);
#pragma unroll
    for (int part = 0; part < (SPLIT ? 2 : 1); ++part) {
        __syncthreads();
        if (mine) {
#pragma unroll
            for (int i = 0; i < kTP2; ++i)
#pragma unroll
                for (int j = 0; j < kTQ2; ++j) {
                    const int q = kWaveRowsQ * qw + 16 * j + r, p = 128 * pw + 16 * i + c;
                    f32x4_t v = acc[i][j] * unit;
                    if constexpr (MODE == kSquare) {
                        // (an operand's multiple that is no f16, or the second of two steps')
                        auto plus = [&](const Pair &from, float by) {
                            const int64_t e = tile + (int64_t)q * ld + p;
                            const f16x4_t h = *(const f16x4_t *)(from.hi + e);
                            f16x4_t lo = {};
                            if constexpr (SPLIT) lo = *(const f16x4_t *)(from.lo + e);
#pragma unroll
                            for (int u = 0; u < 4; ++u) v[u] = fmaf(by, (float)h[u] + (float)lo[u], v[u]);
                        };
                        if (o.E1.hi) plus(o.E1, o.c1);
                        if (o.E2.hi) plus(o.E2, o.c2);
                        if (ti == tj && kWaveRowsQ * qw + 16 * j == 128 * pw + 16 * i) {
#pragma unroll
                            for (int u = 0; u < 4; ++u) v[u] += r == c + u && ti * kTile + q < o.s ? o.diag : 0.0f;
                        }
                    }
                    if constexpr (MODE == kLast) {
                        v *= o.out;
                        *(uint2 *)(t + q * kPitch16 + p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                    } else {
                        f16x4_t w;
#pragma unroll
                        for (int u = 0; u < 4; ++u) w[u] = part ? part_lo(v[u], part_hi(v[u])) : part_hi(v[u]);
                        *(f16x4_t *)(t + q * kPitch16 + p) = w;
                    }
                }
        }
        __syncthreads();
        f16_t *dst = part ? o.dst.lo : o.dst.hi;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int h = b >> 1, g = b & 1;
            if (!wanted(h, g)) continue;
            const f16_t *from = t + kSide * (h * kPitch16 + g);
            // (the mirror image, or what a tall G's update is: through the transposing reads, of 16 columns, 32 rows of a wave's at a time)
            auto across = [&](int k, int &q) {
                q = 32 * k + 2 * c;
                const f16_t *at = from + (q + (r >> 2)) * kPitch16 + 16 * wave + (r & 3) * 4;
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at));
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + 4 * kPitch16));
                return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            if constexpr (MODE == kLast) {
                const int q0 = (2 * ti + h) * kSide, p0 = (2 * tj + g) * kSide;
                bf16_t *out = (bf16_t *)o.O + m * o.s * o.l;
                // eight values of a row of `n`, from element i on
                auto put = [&](bf16_t *row, int i, int n, const s16x8_t &w) {
                    typedef s16x8_t any_t __attribute__((aligned(2)));
                    if (i + 8 <= n) *(any_t *)(row + i) = w;
                    else {
#pragma unroll
                        for (int u = 0; u < 8; ++u)
                            if (i + u < n) row[i + u] = (bf16_t)w[u];
                    }
                };
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (o.transposed) {
                        int q;
                        const s16x8_t w = across(k, q);
                        const int p = p0 + 16 * wave + r;
                        if (p < o.l) put(out + (int64_t)p * o.s, q0 + q, o.s, w);
                    } else {
                        const int e = threadIdx.x + kThreads2 * k, row = e >> 4, col = (e & 15) * 8;
                        if (q0 + row < o.s) put(out + (int64_t)(q0 + row) * o.l, p0 + col, o.l, *(const s16x8_t *)(from + row * kPitch16 + col));
                    }
                }
                continue;
            }
            f16_t *to = dst + tile + (int64_t)h * kSide * ld + g * kSide;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e = threadIdx.x + kThreads2 * k, row = e >> 4, col = (e & 15) * 8;
                *(f16x8_t *)(to + (int64_t)row * ld + col) = *(const f16x8_t *)(from + row * kPitch16 + col);
            }
            if (!kSq || 2 * tj + g == 2 * ti + h) continue;
            f16_t *mirror = dst + tile_at<MODE, kSide>(o, m, 2 * tj + g, 2 * ti + h, ld) + (int64_t)(16 * wave + r) * ld;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                int q;
                const s16x8_t w = across(k, q);
                *(s16x8_t *)(mirror + q) = w;
            }
        }
    }
}

// The others (X's 8 bits, f32 results): two blocks of 128 x 128 at a time, to four waves each, f32 in LDS.  `blocks`: of a row of
// results.
template <int MODE, bool SPLIT, typename OUT>
__device__ __forceinline__ void finish_tile(const Product &o, int64_t m, int ti, int tj, int blocks, const Acc2 &acc, char *lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pw = wave & 1, qw = wave >> 1, side = wave >> 2, tid = threadIdx.x & 255;
    float *mine = (float *)(lds + side * kLdsTile);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int ci = 2 * ti + h, cj = 2 * tj + side;
        const bool wanted = ci < o.sp / kSide && cj < blocks;
        __syncthreads();
        if ((qw >> 1) == h) put_sums<kSide>(acc, 0, 64 * (qw & 1), (float *)(lds + pw * kLdsTile));
        __syncthreads();
        if (wanted) finish_rows<MODE, SPLIT, kSide, OUT>(o, m, ci, cj, mine, tid);
        if constexpr (MODE == kLast) __syncthreads();
        if (wanted) finish_rest<MODE, SPLIT, kSide, OUT>(o, m, ci, cj, mine, tid);
    }
}

// tile t of a lower half, row by row
__device__ __forceinline__ void lower_half(int t, int &ti, int &tj) {
    int i = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    while (i * (i + 1) / 2 > t) --i;
    ti = __builtin_amdgcn_readfirstlane(i);
    tj = __builtin_amdgcn_readfirstlane(t - i * (i + 1) / 2);
}

// X X^T: 256 x 256, the lower half of them.  Its k is the long side and its results are few: the tile loop with the fewest loads.
template <bool SPLIT> __global__ void __launch_bounds__(kThreads2, kMinWavesPerSimd) ortho_gram_kernel(Product o, int64_t matrices) {
    extern __shared__ __align__(1024) char lds[];
    const int64_t at = xcd_share(blockIdx.x, gridDim.x), m = at / o.ntiles;
    int ti, tj;
    lower_half((int)(at - m * o.ntiles), ti, tj);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pw = wave & 1, qw = wave >> 1;
    constexpr int PARTS = SPLIT ? 3 : 1;
    const int64_t xs = (int64_t)o.sp * o.lp, end = matrices * xs;
    const int64_t po = m * xs + (int64_t)tj * kTile * o.lp, qo = m * xs + (int64_t)ti * kTile * o.lp;
    const int nw = o.lp / kBK3;
    RowsOp<PARTS> P, Q;
    P.init(o.P.hi + po, o.P.lo + po, (uint64_t)(end - po) * 2, 2 * o.lp, nw, 0, 128 * pw);
    Q.init(o.P.hi + qo, o.P.lo + qo, (uint64_t)(end - qo) * 2, 2 * o.lp, nw, 1, kWaveRowsQ * qw);
    Acc2 acc;
    zero_acc2(acc);
    mfma_mainloop3<true>(acc, PARTS * nw, P, Q, lds);
    finish_rounded<kGram, SPLIT>(o, m, ti, tj, o.sp / kSide, acc, lds);
}

// The other products.  Tiles of symmetric results are the lower half of them, of others a column of tiles after the other: they share X's
// columns.
template <int MODE, bool SPLIT, typename OUT> __global__ void __launch_bounds__(kThreads2, kMinWavesPerSimd) ortho_product_kernel(Product o, int64_t matrices) {
    extern __shared__ __align__(1024) char lds[];
    const int64_t at = xcd_share(blockIdx.x, gridDim.x), m = at / o.ntiles;
    const int t = (int)(at - m * o.ntiles);
    int ti, tj;
    if constexpr (MODE == kSquare) lower_half(t, ti, tj);
    else {
        const int ni = (o.sp + kTile - 1) / kTile;
        tj = __builtin_amdgcn_readfirstlane(t / ni);
        ti = __builtin_amdgcn_readfirstlane(t - t / ni * ni);
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pw = wave & 1, qw = wave >> 1;
    const int ldp = MODE == kSquare ? o.sp : o.lp;
    const int64_t ps = (int64_t)o.sp * ldp, qs = (int64_t)o.sp * o.sp, po = m * ps + (int64_t)tj * kTile, qo = m * qs + (int64_t)ti * kTile;
    ColumnsOp P, Q;
    P.init(o.P.hi + po, o.P.lo + po, (uint64_t)(matrices * ps - po) * 2, 2 * ldp, o.sp / 32, SPLIT ? 0 : -1, 128 * pw);
    Q.init(o.Q.hi + qo, o.Q.lo + qo, (uint64_t)(matrices * qs - qo) * 2, 2 * o.sp, o.sp / 32, SPLIT ? 1 : -1, kWaveRowsQ * qw);
    Acc2 acc;
    zero_acc2(acc);
    multiply_columns(acc, o.passes, P, Q, (ti * kTile + kWaveRowsQ * qw) / 32, o.own, o.own_lo, lds);
    if constexpr (MODE == kSquare || MODE == kStep || (MODE == kLast && !SPLIT)) finish_rounded<MODE, SPLIT>(o, m, ti, tj, ldp / kSide, acc, lds);
    else finish_tile<MODE, SPLIT, OUT>(o, m, ti, tj, ldp / kSide, acc, lds);
}

// ---- few tiles ----
// Where tiles of 256 would leave most of the card idle, a work-group takes 64 x 64, in windows of 64 k.  Its time is latencies, which other
// work-groups on the compute unit hide better than its own windows: with two of them in 64 KB each, four windows (two with both parts of the
// operands), one 2048 x 2048 to bf16 took 454 us and three 1000 x 501 139, with one in 128 KB 650 and 159; with four in 32 KB
// where products have more than 256 tiles, 392 and 138.  X X^T, whose k is the long side, is cut into parts that are joined by a launch of
// their own.
constexpr int kSmall = 64;
constexpr int kSmallWin = kSmall * kBK3 * 2;     // 8 KB: 64 k of one part of an operand

// 64 k-rows of 64 features; 32-byte group g of k-row k sits at g ^ (k & 3)
struct SmallTr {
    int voff, step, at;
    __device__ __forceinline__ void init(int ld, int wave_base) {
        const int w = threadIdx.x >> 6, lane = lane_id(), row = 8 * w + (lane >> 3);
        voff = row * ld + ((lane & 7) ^ ((row & 3) << 1)) * 16;
        step = 32 * ld;
        const int b = lane >> 4, i = lane & 15, k = 8 * b + (i >> 2);
        at = k * 128 + (((wave_base >> 4) ^ (k & 3)) << 5) + (i & 3) * 8;
    }
    __device__ __forceinline__ static uint32_t advance(int ld) { return 64u * ld; }
    __device__ __forceinline__ bf16x8_t frag(const char *win, int t, int u) const {
        const char *p = win + u * (kSmallWin / 2) + (at ^ (t << 5));
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p + 4 * 128));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// 64 rows of 64 k, as KcLoad
struct SmallKc {
    int voff, step;
    KcFrag16 fr;
    __device__ __forceinline__ void init(int ld, int wave_base) {
        const int w = threadIdx.x >> 6, lane = lane_id(), row = 8 * w + (lane >> 3);
        voff = row * ld + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        step = 32 * ld;
        fr.init(wave_base, lane);
    }
    __device__ __forceinline__ static uint32_t advance(int) { return kBK3 * 2; }
    __device__ __forceinline__ bf16x8_t frag(const char *win, int t, int u) const { return fr.read(win, t, u); }
};
template <class L> __device__ __forceinline__ void small_issue(const L &l, const char *base, int ld, int J, uint32_t win) {
    const rsrc_t r = src_rsrc_inside(Src{base, 0, L::advance(ld)}, J);
    const int w = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < 2; ++i) lds_load16_soff(r, win + 1024 * (w + 4 * i), l.voff, i * l.step);
}

// windows first .. first + n - 1 of P and Q; 4 waves of 32 x 32
template <bool SPLIT, int BUF, class PL, class QL>
__device__ __forceinline__ void multiply_small(f32x4_t (&acc)[2][2], int first, int n, const PL &pl, const Pair &P, int ldp, const QL &ql, const Pair &Q,
                                               int ldq, int own_at, f16_t own, f16_t own_lo, char *lds) {
    constexpr int kParts = SPLIT ? 2 : 1, kBuf = BUF / kParts, kBytes = 2 * kParts * kSmallWin, kEach = 4 * kParts;   // loads of a wave to a window
    const uint32_t at = lds_addr(lds);
    auto issue = [&](int w) {
        const uint32_t to = at + w % kBuf * kBytes;
        small_issue(pl, (const char *)P.hi, ldp, first + w, to);
        small_issue(ql, (const char *)Q.hi, ldq, first + w, to + kParts * kSmallWin);
        if constexpr (SPLIT) {
            small_issue(pl, (const char *)P.lo, ldp, first + w, to + kSmallWin);
            small_issue(ql, (const char *)Q.lo, ldq, first + w, to + 3 * kSmallWin);
        }
    };
    const int ahead = n < kBuf - 1 ? n : kBuf - 1;
    for (int w = 0; w < ahead; ++w) issue(w);
    // the small products, and the operand's own multiple, which is the most of the result: what is added to it is rounded to its last place
    f32x4_t part[2][2] = {}, large[2][2] = {};
    for (int w = 0; w < n; ++w) {
        // (windows w .. w + kBuf - 2 are on their way, if there are as many)
        if (w + kBuf - 2 < n) meet<(kBuf - 2) * kEach>();
        else meet();
        if (w + kBuf - 1 < n) issue(w + kBuf - 1);
        const char *pw = lds + w % kBuf * kBytes, *qw = pw + kParts * kSmallWin;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8_t p[2], q[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                p[i] = pl.frag(pw, i, u);
                q[i] = ql.frag(qw, i, u);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = MfmaF16::run(p[i], q[j], acc[i][j]);
            const bool mine = 2 * (first + w) + u == own_at;      // (32 k and 32 rows)
            if (mine) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8_t e = unit_part(lane_id(), j, own), el = unit_part(lane_id(), j, own_lo);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        part[i][j] = MfmaF16::run(p[i], el, part[i][j]);
                        large[i][j] = MfmaF16::run(p[i], e, large[i][j]);
                    }
                }
            }
            if constexpr (SPLIT) {
                bf16x8_t pl2[2], ql2[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    pl2[i] = pl.frag(pw + kSmallWin, i, u);
                    ql2[i] = ql.frag(qw + kSmallWin, i, u);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        part[i][j] = MfmaF16::run(pl2[i], q[j], part[i][j]);
                        part[i][j] = MfmaF16::run(p[i], ql2[j], part[i][j]);
                        if (mine) part[i][j] = MfmaF16::run(pl2[i], unit_part(lane_id(), j, own), part[i][j]);
                    }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = large[i][j] + (acc[i][j] + part[i][j]);
    meet();
}

// kGram: `cut` parts of the windows to a tile; with more than one, sums go to `parts`, [matrix][tile][part][64 x 64]
template <int MODE, bool SPLIT, int BUF, typename OUT> __global__ void __launch_bounds__(256, BUF == 2 ? 4 : 2) ortho_small_kernel(Product o, int cut, float *__restrict__ parts) {
    extern __shared__ __align__(1024) char lds[];
    const int64_t at = MODE == kGram ? blockIdx.x / cut : blockIdx.x, m = at / o.ntiles;
    const int t = (int)(at - m * o.ntiles), piece = MODE == kGram ? (int)(blockIdx.x - at * cut) : 0;
    int ti, tj;
    if constexpr (MODE == kGram || MODE == kSquare) lower_half(t, ti, tj);
    else {
        const int ni = o.sp / kSmall;
        tj = t / ni;
        ti = t - tj * ni;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p0 = 32 * (wave & 1), q0 = 32 * (wave >> 1);
    const int64_t xs = (int64_t)o.sp * o.lp, as = (int64_t)o.sp * o.sp;
    auto from = [](const Pair &p, int64_t e) { return Pair{p.hi + e, p.lo + e}; };
    f32x4_t acc[2][2] = {};
    SmallKc ql;
    if constexpr (MODE == kGram || MODE == kSquare) {
        const int ld = MODE == kGram ? o.lp : o.sp, nw = ld / kBK3, w0 = (int)((int64_t)nw * piece / cut), w1 = (int)((int64_t)nw * (piece + 1) / cut);
        const int64_t base = m * (MODE == kGram ? xs : as);
        SmallKc pl;
        pl.init(2 * ld, p0);
        ql.init(2 * ld, q0);
        multiply_small<SPLIT, BUF>(acc, w0, w1 - w0, pl, from(o.P, base + (int64_t)tj * kSmall * ld), 2 * ld, ql,
                              from(MODE == kGram ? o.P : o.Q, base + (int64_t)ti * kSmall * ld), 2 * ld, MODE == kGram ? -1 : (ti * kSmall + q0) / 32, o.own,
                              o.own_lo, lds);
    } else {
        SmallTr pl;
        pl.init(2 * o.lp, p0);
        ql.init(2 * o.sp, q0);
        multiply_small<SPLIT, BUF>(acc, 0, o.sp / kBK3, pl, from(o.P, m * xs + (int64_t)tj * kSmall), 2 * o.lp, ql,
                              from(o.Q, m * as + (int64_t)ti * kSmall * o.sp), 2 * o.sp, (ti * kSmall + q0) / 32, o.own, o.own_lo, lds);
    }
    if (MODE == kGram && cut > 1) {
        float *to = parts + (int64_t)blockIdx.x * (kSmall * kSmall) + threadIdx.x * 16;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) *(f32x4_t *)(to + 8 * i + 4 * j) = acc[i][j];
        return;
    }
    put_sums<kSmall>(acc, p0, q0, (float *)lds);
    __syncthreads();
    finish_rows<MODE, SPLIT, kSmall, OUT>(o, m, ti, tj, (float *)lds, threadIdx.x);
    __syncthreads();
    finish_rest<MODE, SPLIT, kSmall, OUT>(o, m, ti, tj, (float *)lds, threadIdx.x);
}

// the parts of a tile of X X^T, in their order
template <bool SPLIT> __global__ void __launch_bounds__(256) ortho_join_kernel(Product o, int cut, const float *__restrict__ parts) {
    __shared__ __align__(16) float sums[kSmall * (kSmall + 4)];
    const int64_t at = blockIdx.x, m = at / o.ntiles;
    int ti, tj;
    lower_half((int)(at - m * o.ntiles), ti, tj);
    const int wave = threadIdx.x >> 6, p0 = 32 * (wave & 1), q0 = 32 * (wave >> 1);
    f32x4_t acc[2][2] = {};
    const float *from = parts + at * cut * (kSmall * kSmall) + threadIdx.x * 16;
#pragma unroll 4
    for (int c = 0; c < cut; ++c, from += kSmall * kSmall)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] += *(const f32x4_t *)(from + 8 * i + 4 * j);
    put_sums<kSmall>(acc, p0, q0, sums);
    __syncthreads();
    finish_rows<kGram, SPLIT, kSmall, float>(o, m, ti, tj, sums, threadIdx.x);
    finish_rest<kGram, SPLIT, kSmall, float>(o, m, ti, tj, sums, threadIdx.x);
}

// ---- the start: |G| and X = G kUnit / (|G| + eps) ----
constexpr int kNormParts = 64;
constexpr int kNormElems = 16384;   // of a part at least

template <typename T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const T *__restrict__ G, int64_t elems, int parts, double *__restrict__ part) {
    const int64_t m = blockIdx.x / parts;
    const int p = (int)(blockIdx.x - m * parts);
    const int64_t per = (elems + parts - 1) / parts, lo = p * per, hi = lo + per < elems ? lo + per : elems;
    const T *g = G + m * elems;
    // (squares of f32 are exact in f64, and neither overflow nor vanish there)
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    int64_t i = lo + threadIdx.x;
    for (; i + 3 * 256 < hi; i += 4 * 256) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const double v = Elem<T>::ld(g + i + u * 256);
            sum[u] = fma(v, v, sum[u]);
        }
    }
    for (; i < hi; i += 256) {
        const double v = Elem<T>::ld(g + i);
        sum[0] = fma(v, v, sum[0]);
    }
    __shared__ double ws[4];
    const double w = wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
    if (lane_id() == 0) ws[threadIdx.x >> 6] = w;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = (ws[0] + ws[1]) + (ws[2] + ws[3]);
}

// An N x N tile of X, a tall G's through LDS.  Rows of G are read in vectors of 16 bytes, at any element's address.
template <int N, typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(const T *__restrict__ G, Product o, int parts, const double *__restrict__ part, double eps,
                                                          bool split, int32_t *__restrict__ status) {
    extern __shared__ __align__(1024) char lds[];
    __shared__ double inv_s;
    float *tile = (float *)lds;
    const int nj = o.lp / N, per = o.sp / N * nj;
    const int64_t m = blockIdx.x / per;
    const int t = (int)(blockIdx.x - m * per), i0 = t / nj * N, j0 = t % nj * N;
    if (threadIdx.x < kWave) {
        const double s = wave_sum((int)threadIdx.x < parts ? part[m * parts + threadIdx.x] : 0.0);
        if (threadIdx.x == 0) {
            const double n = sqrt(s) + eps;
            inv_s = n == 0.0 ? 0.0 : isfinite(s) ? (double)kUnit / n : (double)NAN;
            if (!isfinite(s) && t == 0 && status) atomicOr(status, R3_DATA_NONFINITE);
        }
    }
    const T *g = G + m * (int64_t)o.s * o.l;
    const int r0 = o.transposed ? j0 : i0, c0 = o.transposed ? i0 : j0, rows = o.transposed ? o.l : o.s, cols = o.transposed ? o.s : o.l;
    constexpr int kVec = Row<T>::kVec, kEach = N * N / kVec / 256, kRow = N / kVec;
    float x[kEach][kVec];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int e = threadIdx.x + 256 * k, r = e / kRow, c = e % kRow * kVec;
        const T *at = g + (int64_t)(r0 + r) * cols + c0 + c;
        const bool row = r0 + r < rows;
        if (row && c0 + c + kVec <= cols) Row<T>::unpack(Row<T>::load(at), x[k]);
        else {
#pragma unroll
            for (int u = 0; u < kVec; ++u) x[k][u] = row && c0 + c + u < cols ? Elem<T>::ld(at + u) : 0.0f;
        }
    }
    __syncthreads();
    const double inv = inv_s;
    // (in 64 bits: 1 / |G| may be beyond f32's range)  Beyond G's rows and columns X is 0 whatever the norm is.
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int e = threadIdx.x + 256 * k, r = e / kRow, c = e % kRow * kVec;
#pragma unroll
        for (int u = 0; u < kVec; ++u) {
            x[k][u] = r0 + r < rows && c0 + c + u < cols ? (float)((double)x[k][u] * inv) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kVec; u += 4) *(f32x4_t *)(tile + sums_at<N>(r, c + u)) = f32x4_t{x[k][u], x[k][u + 1], x[k][u + 2], x[k][u + 3]};
    }
    __syncthreads();
    const int64_t base = m * (int64_t)o.sp * o.lp + (int64_t)i0 * o.lp + j0;
#pragma unroll 2
    for (int k = 0; k < N * N / 8 / 256; ++k) {
        const int e = threadIdx.x + 256 * k, r = e / (N / 8), c = e % (N / 8) * 8;
        float v[8];
        if (o.transposed) read_down<N>(tile, c, r, v);
        else read_along<N>(tile, r, c, v);
        if (split) put8<kRest16>(o.dst, base + (int64_t)r * o.lp + c, v);
        else put8<kRest8>(o.dst, base + (int64_t)r * o.lp + c, v);
    }
}

// Tiles of 64 x 64 up to some twelve of X's to a compute unit, sixteen where products are three (us a call, 64 x 64 | 256 x 256; bf16
// results: 30 x 300 x 700 235 | 346, 2 x 2048 x 2048 733 | 868, 16 x 512 x 1024 317 | 412, 24 x 444 | 428, 32 x 579 | 451, 64 x 256 x 512
// 222 | 288, 100 x 316 | 312, 128 x 388 | 335, 40 x 385 x 900 620 | 530, 1 x 4096 x 4096 2377 | 1674; f32: 1 x 2048 x 2048 840 | 2445, 24 x
// 512 x 1024 805 | 1034, 32 x 1079 | 1060, 10 x 768 x 2048 1090 | 1411, 128 x 256 x 512 738 | 722).
bool small_tiles(int64_t batch, int64_t s, int64_t l, bool split) {
    return batch * ((s + kSmall - 1) / kSmall) * ((l + kSmall - 1) / kSmall) <= (split ? 4000 : 3000);
}

struct Plan {
    int s, l, sp, lp, parts;
    int64_t chunk;             // matrices at a time
    size_t norm, X, Y, A, B, C, parts_at, total;
    bool narrow;               // r3_ortho_narrow.hip's, with X's place for all of its workspace
    bool split, small;         // split: products of pairs; small: tiles of 64
    int cut;                   // parts of X X^T
};

Plan plan(int64_t batch, int64_t rows, int64_t cols, int dtype_out) {
    Plan p;
    p.s = (int)(rows < cols ? rows : cols);
    p.l = (int)(rows < cols ? cols : rows);
    p.narrow = p.s <= kNarrowSide;
    p.split = dtype_out == R3_F32;
    p.small = !p.narrow && small_tiles(batch, p.s, p.l, p.split);
    const int side = p.small ? kSmall : kSide;
    p.sp = (p.s + side - 1) / side * side;
    p.lp = (p.l + side - 1) / side * side;
    const int64_t elems = rows * cols;
    p.parts = (int)((elems + kNormElems - 1) / kNormElems);
    if (p.parts > kNormParts) p.parts = kNormParts;
    const size_t x = (size_t)p.sp * p.lp * (p.split ? 4 : 3), a = (size_t)p.sp * p.sp * (p.split ? 4 : 2);   // of a matrix: X or Y, A, B or C
    const size_t most = (size_t)4 << 30;
    const int64_t fit = (int64_t)(most / (2 * x + 3 * a));
    p.chunk = fit < 1 ? 1 : fit < batch ? fit : batch;
    p.cut = 1;
    const int nt = p.sp / kSmall, tiles = nt * (nt + 1) / 2, nw = p.lp / kBK3;
    // A work-group to a compute unit, at least four windows to a part (of pairs) or eight; up to 24 the join costs more (3 x 1000 x 501 to
    // bf16, 16 windows, 123 us uncut, 136 in two; 5 x 200 x 1500, 24, 119 | 122 in three; 1 x 512 x 2048, 32, 133 in four, 138 in two).
    if (p.small && (p.split || nw > 24)) p.cut = (int)std::max<int64_t>(1, std::min<int64_t>(nw / (p.split ? 4 : 8), 256 / (tiles * p.chunk)));
    size_t o = 0;
    // (a tile of 256 columns may read 128 columns past a matrix's last)
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes + 2 * kSide, 256); return at; };
    p.norm = take((size_t)batch * p.parts * sizeof(double));
    if (p.narrow) {
        p.X = take(ortho_narrow_ws_bytes(batch, p.s, p.l));
        p.total = o;
        return p;
    }
    p.X = take(x * p.chunk);
    p.Y = take(x * p.chunk);
    p.A = take(a * p.chunk);
    p.B = take(a * p.chunk);
    p.C = take(a * p.chunk);
    p.parts_at = take(p.cut > 1 ? (size_t)p.chunk * tiles * p.cut * kSmall * kSmall * sizeof(float) : 0);
    p.total = o;
    return p;
}

// Steps taken together: X'' = Q X with Q = (a + b A' + c A' A') (a + b A + c A A) and A' = (a + b A + c A A)^2 A, without X' between them:
// five products of s x s instead of two, and a product with X and an X X^T less.  On small tiles that is as many launches, which are what
// counts there, and steps stay apart.  Else for f32 results wherever two steps are left; for bf16 ones at the start alone, where it costs
// no exactness: later a rounding of X enters the second product times a^2.  (Simulated with 11 bits of X's rest, Frobenius norm, five
// steps, random 256 x 768 / falling singular values / rank 3: apart 1.1e-3 / 8e-4 / 3.0e-3, the first two together the same, the first two pairs
// 1.3e-3 / 1.6e-3 / 9e-3.)
bool two_together(int step, int steps, bool all, bool pairs) { return pairs && ortho_together(step, steps, all); }

// Whether every element stays in (-15, 15), so that times kUnit it is an f16: a matrix's are at most its largest singular value, that of X
// at most 1 at the start and then what the quintic makes of it.  At equidistant points: between two of 2 n over (-r, r) a polynomial of
// degree d is at most d^2 (d^2 - 1) / 24 n^2 of its maximum beyond them, 1.3 % at degree 6 and 64 points, 21 % at degree 24 (two steps) and 256.
bool in_range(int steps, const float *q, bool all, bool pairs) {
    const double a = q[0], b = q[1], c = q[2];
    // the largest of |values| (that are finite: |q| is below 2^128)
    auto more = [](double v, double &most) {
        v = v < 0.0 ? -v : v;
        most = v > most ? v : most;
    };
    double r = 1.0;
    for (int k = 0; k < steps;) {
        const bool two = two_together(k, steps, all, pairs);
        const double out = ortho_apart(k, steps, q) * (two ? ortho_apart(k + 1, steps, q) : 1.0);
        double most = 0.0, next = 0.0;
        for (int i = 0; i <= 64; ++i) {
            const double x = r * i / 64, y = x * x, P = a + y * (b + y * c);
            more(x, most);
            more(y, most);
            more(two ? P - a : P - out, most);
            more(x * P, next);
        }
        most *= 1.02;
        next *= 1.02;
        if (two) {
            double pair = 0.0, last = 0.0;
            for (int i = 0; i <= 256; ++i) {
                const double x = r * i / 256, y = x * x, P = a + y * (b + y * c), y1 = x * P * (x * P), P1 = a + y1 * (b + y1 * c);
                more(P * y, pair);
                more(y1, pair);
                more(P1 - a, pair);
                more(P * P1 - out, pair);
            }
            for (int i = 0; i <= 64; ++i) {
                const double x = next * i / 64, y = x * x;
                more(x * (a + y * (b + y * c)), last);
            }
            more(pair * 1.25, most);
            next = last * 1.02;
        }
        more(out, most);
        if (!(most < 15.0 && next < 15.0)) return false;
        r = next;
        k += two ? 2 : 1;
    }
    return true;
}

template <int BUF> struct Buffers { static constexpr int kBuf = BUF, kLds = 2 * BUF * kSmallWin; };

template <int NT = 256, class K, class... A> hipError_t launch(K k, int64_t grid, int lds, hipStream_t s, const A &...args) {
    (void)hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    k<<<(unsigned)grid, NT, lds, s>>>(args...);
    return hipGetLastError();
}

// bf16 results: hi hi; f32 ones: pairs.
template <bool SPLIT>
hipError_t iterate(const Plan &p, Product o, Pair X, Pair Y, Pair A, Pair B, Pair C, float *parts, int64_t matrices, int steps, const float *coef,
                   float scale, bool pairs, hipStream_t s) {
    typedef typename std::conditional<SPLIT, float, bf16_t>::type OUT;
    const int side = p.small ? kSmall : kTile, ns = (o.sp + side - 1) / side, half = ns * (ns + 1) / 2, step_tiles = ns * ((o.lp + side - 1) / side);
    const float a = coef[0], b = coef[1], c = coef[2];
    const Pair none = {nullptr, nullptr};
    float *no_parts = nullptr;
    o.passes = SPLIT ? 3 : 1;
    hipError_t e = hipSuccess;
    // 64 x 64 tiles: four windows, or two where that puts more of them on a compute unit
    auto small = [&](auto mode, auto type, int64_t grid, int cut, float *to) {
        constexpr int MODE = decltype(mode)::value;
        typedef decltype(type) T;
        auto by = [&](auto b) {
            typedef decltype(b) W;
            return launch(ortho_small_kernel<MODE, SPLIT, W::kBuf, T>, grid, W::kLds, s, o, cut, to);
        };
        if constexpr (!SPLIT) {
            if (grid > 256) return by(Buffers<2>{});
        }
        return by(Buffers<4>{});
    };
    auto gram = [&](Pair to) {
        o.ntiles = half;
        o.P = X; o.dst = to;
        if (e != hipSuccess) return;
        if (!p.small) e = launch<kThreads2>(ortho_gram_kernel<SPLIT>, matrices * half, 2 * kLdsTile, s, o, matrices);
        else e = small(std::integral_constant<int, kGram>{}, 0.0f, matrices * half * p.cut, p.cut, parts);
        if (e == hipSuccess && p.cut > 1) e = launch(ortho_join_kernel<SPLIT>, matrices * half, 0, s, o, p.cut, (const float *)parts);
    };
    auto set_own = [&](double v) {
        o.own = (f16_t)(float)(v * kUnit);
        o.own_lo = (f16_t)(float)(v * kUnit - (double)(float)o.own);
    };
    // to = cd q from + c1 from + c2 e2 + diag
    auto square = [&](Pair to, float cd, Pair q, Pair from, float c1, float c2, Pair e2, double diag) {
        o.ntiles = half;
        o.Q = q; o.P = from; o.E2 = e2; o.dst = to;
        // (a quotient that is no f16: the matrix is read again)
        const bool own = std::fabs((double)c1) < 15.0 * std::fabs((double)cd);
        set_own(own ? (double)c1 / cd : 0.0);
        o.E1 = own ? none : from;
        o.cd = cd; o.c1 = c1; o.c2 = c2; o.diag = (float)(diag * kUnit);
        if (e != hipSuccess) return;
        e = p.small ? small(std::integral_constant<int, kSquare>{}, 0.0f, matrices * half, 1, no_parts)
                    : launch<kThreads2>(ortho_product_kernel<kSquare, SPLIT, float>, matrices * half, 2 * kLdsTile, s, o, matrices);
    };
    for (int k = 0; k < steps;) {
        const bool two = two_together(k, steps, SPLIT, pairs);
        double out_of = ortho_apart(k, steps, coef);
        Pair q = B;
        gram(A);
        if (two) {
            out_of *= ortho_apart(k + 1, steps, coef);
            square(B, c, A, A, b, 0.0f, none, 0.0);                             // B = b A + c A A
            square(C, 1.0f, B, A, a, 0.0f, none, 0.0);                          // C = (a + B) A
            square(A, 1.0f, B, C, a, 0.0f, none, 0.0);                          // A' = (a + B) C
            square(C, c, A, A, b, 0.0f, none, 0.0);                             // B' = b A' + c A' A'
            square(A, 1.0f, C, B, a, a, C, (double)a * a - out_of);             // Q = (a + B') (a + B)
            q = A;
        } else {
            square(B, c, A, A, b, 0.0f, none, (double)a - out_of);
        }
        k += two ? 2 : 1;
        o.ntiles = step_tiles;
        // (pairs have X's lo in their products; else 8 bits of it count while three steps and more are left)
        const bool had = !SPLIT && steps - (k - (two ? 2 : 1)) > 2, keeps = !SPLIT && steps - k > 2;
        o.Q = q; o.P = X; o.E1 = had ? X : none; o.dst = SPLIT || keeps ? Y : Pair{Y.hi, nullptr};
        set_own(out_of);
        o.c1 = (float)out_of;
        o.out = scale / kUnit;
        const int64_t grid = matrices * step_tiles;
        if (e != hipSuccess) return e;
        auto step = [&](auto mode) {
            constexpr int MODE = decltype(mode)::value;
            return p.small ? small(mode, 0.0f, grid, 1, no_parts)
                           : launch<kThreads2>(ortho_product_kernel<MODE, SPLIT, float>, grid, 2 * kLdsTile, s, o, matrices);
        };
        if (k == steps) {
            e = p.small ? small(std::integral_constant<int, kLast>{}, OUT{}, grid, 1, no_parts)
                        : launch<kThreads2>(ortho_product_kernel<kLast, SPLIT, OUT>, grid, 2 * kLdsTile, s, o, matrices);
        } else if constexpr (SPLIT) {
            e = step(std::integral_constant<int, kStep>{});
        } else {
            e = had || keeps ? step(std::integral_constant<int, kStepLow>{}) : step(std::integral_constant<int, kStep>{});
        }
        std::swap(X, Y);
    }
    return e;
}

}  // namespace

size_t orthogonalize_ws_bytes(int64_t batch, int64_t rows, int64_t cols, int dtype_out) { return plan(batch, rows, cols, dtype_out).total; }

bool orthogonalize_in_range(int steps, const float *coef) { return in_range(steps, coef, false, false); }

hipError_t launch_orthogonalize(int64_t batch, int64_t rows, int64_t cols, int dtype_in, const void *G, int dtype_out, void *out, int steps,
                                const float *coef, float eps, float scale, int32_t *status, void *ws, hipStream_t s) {
    ProfScope ps(PROF_ORTHO, s);
    const Plan p = plan(batch, rows, cols, dtype_out);
    char *base = (char *)ws;
    double *part = (double *)(base + p.norm);
    const int64_t elems = rows * cols;
    const size_t eb = dtype_in == R3_BF16 ? 2 : 4, ob = dtype_out == R3_BF16 ? 2 : 4;
    auto norms = [&](const char *g, int64_t nm, double *to) {
        if (dtype_in == R3_BF16) ortho_norm_kernel<bf16_t><<<(unsigned)(nm * p.parts), 256, 0, s>>>((const bf16_t *)g, elems, p.parts, to);
        else ortho_norm_kernel<float><<<(unsigned)(nm * p.parts), 256, 0, s>>>((const float *)g, elems, p.parts, to);
        return hipGetLastError();
    };
    if (p.narrow) {
        constexpr int64_t kMost = 1 << 17;      // matrices to a launch: 2^31 threads at the most
        for (int64_t m0 = 0; m0 < batch; m0 += kMost) {
            const hipError_t e = norms((const char *)G + (size_t)m0 * elems * eb, std::min(kMost, batch - m0), part + m0 * p.parts);
            if (e != hipSuccess) return e;
        }
        NarrowCall c = {};
        c.batch = batch; c.s = p.s; c.l = p.l; c.steps = steps; c.norms = p.parts;
        c.transposed = rows > cols;
        c.pairs = in_range(steps, coef, dtype_out == R3_BF16, true);
        c.G = G; c.O = out; c.ws = base + p.X;
        c.norm = part;
        c.coef = coef;
        c.eps = eps; c.scale = scale;
        c.status = status;
        return launch_ortho_narrow(c, dtype_in, dtype_out, s);
    }
    // (the matrices between two steps have larger elements than those of one: other coefficients may have room for single ones alone)
    const bool pairs = !p.small && in_range(steps, coef, p.split, true);
    for (int64_t m0 = 0; m0 < batch; m0 += p.chunk) {
        const int64_t nm = batch - m0 < p.chunk ? batch - m0 : p.chunk;
        const int64_t xs = (int64_t)p.sp * p.lp * p.chunk, as = (int64_t)p.sp * p.sp * p.chunk;
        Product o = {};
        o.s = p.s; o.l = p.l; o.sp = p.sp; o.lp = p.lp;
        o.transposed = rows > cols;
        auto pair = [&](size_t at, int64_t n) { return Pair{(f16_t *)(base + at), (f16_t *)(base + at) + n}; };
        const Pair X = pair(p.X, xs), Y = pair(p.Y, xs), A = pair(p.A, as), B = pair(p.B, as), C = pair(p.C, as);
        o.O = (char *)out + (size_t)m0 * elems * ob;
        o.dst = X;
        const char *g = (const char *)G + (size_t)m0 * elems * eb;
        const int side = p.small ? kSmall : kSide;
        const int64_t ntiles = nm * (p.sp / side) * (p.lp / side);
        hipError_t e = norms(g, nm, part);
        if (e != hipSuccess) return e;
        auto start = [&](auto type) {
            typedef decltype(type) T;
            auto k = p.small ? ortho_start_kernel<kSmall, T> : ortho_start_kernel<kSide, T>;
            e = launch(k, ntiles, side * (side + 4) * 4, s, (const T *)g, o, p.parts, (const double *)part, (double)eps, p.split, status);
        };
        if (dtype_in == R3_BF16) start(bf16_t{});
        else start(float{});
        if (e != hipSuccess) return e;
        auto run = p.split ? iterate<true> : iterate<false>;
        e = run(p, o, X, Y, A, B, C, (float *)(base + p.parts_at), nm, steps, coef, scale, pairs, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace r3
