// Newton-Schulz orthogonalisation of a batch of matrices:  X = G / (|G|_F + eps);  steps times  A = X X^T,  X <- a X + (b A + c A A) X.
// With X = U S V^T a step takes every singular value x to a x + b x^3 + c x^5 and leaves U and V alone.  The short side is the rows
// of X (a tall G is read and written transposed), so that A is s x s; it and its polynomial are symmetric and half their tiles are made.
//
// Numbers.  The matrix instruction's f16 operands, f32 sums.  A step's values are known beforehand: |X|_2 stays below about 1.2, so no
// element of X, A or B = b A + c A A leaves (-16, 16) (the host checks it for other coefficients), and everything is stored times 2^12:
// at best 11 bits, four times bf16's, down to 1.5e-8.  A rounding of X is an error that the coming steps multiply by up to a each (a
// small singular value grows by a, a new one beside it does too), so X is kept as two f16, its rounding and the rounding of the rest; one
// of them enters the products, where the small directions hardly count.  The last two steps' polynomial has a + b + c, what it is for
// singular values of 1, taken out of B and applied to X in f32, so that B's rounding is one of a small matrix.  Relative error of bf16
// results beside their own rounding (1.7e-3): 4e-4 ... 1.0e-3 for matrices with flat and falling spectra; with bf16 operands throughout
// it is 1e-2 ... 4e-2.  For f32 results all of X, A, B are such pairs and products are the three of their parts that count
// (hi lo, lo hi, hi hi): 22 bits, 3e-7 ... 8e-7 where f32 products give 2e-7 ... 5e-7.
#include <cmath>

#include "r3_kernels.h"
#include "r3_mfma2.h"
#include "r3_vec.h"

namespace r3 {
namespace {

typedef _Float16 f16_t;
typedef f16_t f16x4_t __attribute__((ext_vector_type(4)));
typedef f16_t f16x8_t __attribute__((ext_vector_type(8)));

constexpr int kSide = 128;                 // a work-group's tile
constexpr int kWin = kSide * kBK3 * 2;     // 16 KB: 64 k of an operand
constexpr float kUnit = 4096.0f;           // what is stored is times this
constexpr int kPitchF = kSide + 4;         // of a tile of results in LDS
constexpr int kLdsBytes = kSide * kPitchF * 4;   // 66 KB: four windows of operands, or a tile of results
static_assert(kLdsBytes >= 4 * kWin, "");

enum { kGram = 0, kPoly = 1, kStep = 2, kLast = 3 };

struct Pair { f16_t *hi, *lo; };   // lo may be null
struct Ortho {
    int s, l, sp, lp;              // X is s x l in sp x lp, zeros beyond
    int ntiles;                    // of a matrix
    Pair X, Y, A, B;
    float a, b, c, out;            // X' = a X + B X (kStep, kLast: times out); B = a I + b A + c A A (kPoly)
    void *O;
    bool transposed;
};

// one operand's window of 64 k, rows or k-rows of ld bytes; all of them exist
struct KcLoad {
    static constexpr bool kTr = false;
    int voff, step;
    KcFrag16 fr;
    __device__ __forceinline__ void init(int ld, int wave_base) {
        const int w = threadIdx.x >> 6, lane = lane_id(), row = 8 * w + (lane >> 3);
        voff = row * ld + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        step = 32 * ld;
        fr.init(wave_base, lane);
    }
    __device__ __forceinline__ static uint32_t advance(int) { return kBK3 * 2; }   // from window to window
    __device__ __forceinline__ void issue(const Src &src, int J, uint32_t win) const {
        const rsrc_t r = src_rsrc_inside(src, J);
        const int w = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < 4; ++i) lds_load16_soff(r, win + 1024 * (w + 4 * i), voff, i * step);
    }
    __device__ __forceinline__ f16x8_t frag(const char *win, int t, int u) const { return __builtin_bit_cast(f16x8_t, fr.read(win, t, u)); }
};
struct TrLoad {
    static constexpr bool kTr = true;
    int ld;
    DmaTR<128> dma;
    TrFrag16<128> fr;
    __device__ __forceinline__ void init(int ld_, int wave_base) {
        ld = ld_;
        dma.init(ld, 0);
        fr.init(wave_base);
    }
    __device__ __forceinline__ static uint32_t advance(int ld) { return 32u * ld; }   // from half to half
    __device__ __forceinline__ void issue(const Src &src, int J, uint32_t win) const {
        dma.issue(src_rsrc_inside(src, 2 * J), win);
        dma.issue(src_rsrc_inside(src, 2 * J + 1), win + kWin / 2);
    }
    __device__ __forceinline__ f16x8_t frag(const char *win, int t, int u) const {
        return __builtin_bit_cast(f16x8_t, fr.read(win + u * (kWin / 2), t));
    }
};

typedef f32x4_t Acc[4][4];

// All loads of a window have landed and everybody has left the one before, whose place the next loads take.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    window_barrier<0>();
    asm volatile("" ::: "memory");
}

// acc[i][j] += sum over k of P's row p and Q's row q; 4 waves of 64 x 64, as 4 x 4 of 16 x 16.  `parts` 1: hi hi; 3: lo hi, hi lo, hi hi.
template <int PARTS, class PL, class QL>
__device__ __forceinline__ void multiply(Acc &acc, int nw, const PL &pl, const char *phi, const char *plo, uint32_t padv, const QL &ql,
                                         const char *qhi, const char *qlo, uint32_t qadv, char *lds) {
    const uint32_t at = lds_addr(lds);
    int part = 0, J = 0;      // of the next window to load
    auto issue = [&](int buf) {
        const bool plow = PARTS == 3 && part == 0, qlow = PARTS == 3 && part == 1;
        pl.issue(Src{plow ? plo : phi, 0, padv}, J, at + buf * 2 * kWin);
        ql.issue(Src{qlow ? qlo : qhi, 0, qadv}, J, at + buf * 2 * kWin + kWin);
        if (++J == nw) {
            J = 0;
            ++part;
        }
    };
    issue(0);
    for (int w = 0; w < PARTS * nw; ++w) {
        meet();
        if (w + 1 < PARTS * nw) issue((w + 1) & 1);
        const char *pw = lds + (w & 1) * 2 * kWin, *qw = pw + kWin;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f16x8_t p[4], q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = pl.frag(pw, i, u);
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = ql.frag(qw, j, u);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) {
                    const int i = (j & 1) ? 3 - ii : ii;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[i], q[j], acc[i][j], 0, 0, 0);
                }
        }
    }
    meet();
}

__device__ __forceinline__ f16_t part_hi(float v) { return (f16_t)v; }
__device__ __forceinline__ f16_t part_lo(float v, f16_t hi) { return (f16_t)(v - (float)hi); }

// A tile of results in LDS, row q at q kPitchF with its columns' fours exchanged by q / 8, so that eight rows' values of a column, 16 x 4
// of them to a wave, meet at most two at a time in a bank; col is a multiple of 8 (read_down: row).
__device__ __forceinline__ int sums_at(int q, int p) { return q * kPitchF + (p ^ (((q >> 3) & 7) << 2)); }
__device__ __forceinline__ void read_along(const float *sums, int row, int col, float *v) {
    *(f32x4_t *)v = *(const f32x4_t *)(sums + sums_at(row, col));
    *(f32x4_t *)(v + 4) = *(const f32x4_t *)(sums + sums_at(row, col + 4));
}
__device__ __forceinline__ void read_down(const float *sums, int row, int col, float *v) {
    const float *at = sums + sums_at(row, col);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = at[u * kPitchF];
}
// eight values to their place, and what their rounding leaves
template <bool LO> __device__ __forceinline__ void put8(const Pair &dst, int64_t e, const float *v) {
    f16x8_t h, lo;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        h[u] = part_hi(v[u]);
        lo[u] = part_lo(v[u], h[u]);
    }
    *(f16x8_t *)(dst.hi + e) = h;
    if constexpr (LO) *(f16x8_t *)(dst.lo + e) = lo;
}

// where a work-group's number takes it: the groups of an XCD (every eighth) have neighbouring tiles, and so the same matrices in its L2
__device__ __forceinline__ int64_t xcd_share(int64_t id, int64_t n) {
    const int64_t x = id & 7, q = n >> 3, r = n & 7;
    return x * q + (x < r ? x : r) + (id >> 3);
}

template <int MODE, bool SPLIT, typename OUT>
__global__ void __launch_bounds__(256, 2) ortho_tile_kernel(Ortho o) {
    extern __shared__ __align__(1024) char lds[];
    const int64_t at = xcd_share(blockIdx.x, gridDim.x), m = at / o.ntiles;
    const int t = (int)(at - m * o.ntiles);
    int ti, tj;       // tile row and column
    if constexpr (MODE == kGram || MODE == kPoly) {
        ti = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
        while (ti * (ti + 1) / 2 > t) --ti;
        tj = t - ti * (ti + 1) / 2;
    } else {
        const int nj = o.lp / kSide;
        ti = t / nj;
        tj = t - ti * nj;
    }
    ti = __builtin_amdgcn_readfirstlane(ti);
    tj = __builtin_amdgcn_readfirstlane(tj);
    const int64_t xs = (int64_t)o.sp * o.lp, as = (int64_t)o.sp * o.sp;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
    const int p0 = 64 * (wave & 1), q0 = 64 * (wave >> 1);
    Acc acc;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int PARTS = SPLIT ? 3 : 1;
    KcLoad ql;
    if constexpr (MODE == kGram || MODE == kPoly) {
        const Pair in = MODE == kGram ? o.X : o.A;
        const int ldk = MODE == kGram ? o.lp : o.sp;
        const int64_t base = m * (MODE == kGram ? xs : as), ro = base + (int64_t)ti * kSide * ldk, co = base + (int64_t)tj * kSide * ldk;
        KcLoad pl;
        pl.init(2 * ldk, p0);
        ql.init(2 * ldk, q0);
        multiply<PARTS>(acc, ldk / kBK3, pl, (const char *)(in.hi + co), (const char *)(in.lo + co), KcLoad::advance(0), ql,
                        (const char *)(in.hi + ro), (const char *)(in.lo + ro), KcLoad::advance(0), lds);
    } else {
        TrLoad pl;
        pl.init(2 * o.lp, p0);
        ql.init(2 * o.sp, q0);
        const int64_t xo = m * xs + (int64_t)tj * kSide, bo = m * as + (int64_t)ti * kSide * o.sp;
        multiply<PARTS>(acc, o.sp / kBK3, pl, (const char *)(o.X.hi + xo), (const char *)(o.X.lo + xo), TrLoad::advance(2 * o.lp), ql,
                        (const char *)(o.B.hi + bo), (const char *)(o.B.lo + bo), KcLoad::advance(0), lds);
    }
    // The sums through LDS, so that whole lines of X or A are read and written.  A lane's: rows q0 + 16 j + (lane & 15), columns
    // p0 + 16 i + 4 (lane >> 4) .. + 3.
    float *sums = (float *)lds;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *(f32x4_t *)(sums + sums_at(q0 + 16 * j + (lane & 15), p0 + 16 * i + 4 * (lane >> 4))) = acc[i][j] * (1.0f / kUnit);
    __syncthreads();
    constexpr bool kMirror = MODE == kGram || MODE == kPoly;
    const int64_t ld = kMirror ? o.sp : o.lp;
    const int64_t tile = m * (kMirror ? as : xs) + (int64_t)ti * kSide * ld + (int64_t)tj * kSide;
    const Pair dst = MODE == kGram ? o.A : MODE == kPoly ? o.B : o.Y;
    // eight columns of a row to a thread at a time (times kUnit: both operands are)
#pragma unroll 2
    for (int k = 0; k < kSide * kSide / 8 / 256; ++k) {
        const int c = threadIdx.x + 256 * k, r = c >> 4, col = (c & 15) * 8;
        const int64_t e = tile + (int64_t)r * ld + col;
        float v[8], x[8];
        if constexpr (MODE != kGram) {
            const Pair in = MODE == kPoly ? o.A : o.X;
            const f16x8_t h = *(const f16x8_t *)(in.hi + e);
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = (float)h[u];
            if (MODE != kPoly || SPLIT) {
                const f16x8_t lo = *(const f16x8_t *)(in.lo + e);
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] += (float)lo[u];
            }
        }
        read_along(sums, r, col, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if constexpr (MODE == kPoly) {
                v[u] = fmaf(o.c, v[u], o.b * x[u]);
                const int row = ti * kSide + r;
                if (row == tj * kSide + col + u && row < o.s) v[u] += o.a * kUnit;
            } else if constexpr (MODE == kStep || MODE == kLast) {
                v[u] = fmaf(o.a, x[u], v[u]);
                if constexpr (MODE == kLast) v[u] *= o.out;
            }
        }
        if constexpr (MODE == kPoly || MODE == kLast) {
#pragma unroll
            for (int u = 0; u < 8; u += 4) *(f32x4_t *)(sums + sums_at(r, col + u)) = *(const f32x4_t *)(v + u);
        }
        if constexpr (MODE != kLast) put8<MODE == kStep || SPLIT>(dst, e, v);
    }
    if constexpr (MODE == kLast) {
        __syncthreads();
        const int rows = o.transposed ? o.l : o.s, cols = o.transposed ? o.s : o.l;
        const int r0 = (o.transposed ? tj : ti) * kSide, c0 = (o.transposed ? ti : tj) * kSide;
        OUT *out = (OUT *)o.O + m * rows * cols;
        for (int k = 0; k < kSide * kSide / 8 / 256; ++k) {
            const int e = threadIdx.x + 256 * k, r = e >> 4, c = (e & 15) * 8;
            if (r0 + r >= rows || c0 + c >= cols) continue;
            float v[8];
            if (o.transposed) read_down(sums, c, r, v);
            else read_along(sums, r, c, v);
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
    if constexpr (kMirror) {
        if (ti == tj) return;
        __syncthreads();
        // the mirror image: eight rows' values of one column to a thread
        const int64_t mirrored = m * as + (int64_t)tj * kSide * ld + (int64_t)ti * kSide;
#pragma unroll 2
        for (int k = 0; k < kSide * kSide / 8 / 256; ++k) {
            const int c = threadIdx.x + 256 * k, r = c >> 4, col = (c & 15) * 8;
            float v[8];
            read_down(sums, col, r, v);
            put8<SPLIT>(dst, mirrored + (int64_t)r * ld + col, v);
        }
    }
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

// A 128 x 128 tile of X, a tall G's through LDS.  Rows of G are read in vectors of 16 bytes, at any element's address.
template <typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(const T *__restrict__ G, Ortho o, int parts, const double *__restrict__ part, double eps,
                                                          int32_t *__restrict__ status) {
    extern __shared__ __align__(1024) char lds[];
    __shared__ double inv_s;
    float *tile = (float *)lds;
    const int nj = o.lp / kSide, per = o.sp / kSide * nj;
    const int64_t m = blockIdx.x / per;
    const int t = (int)(blockIdx.x - m * per), i0 = t / nj * kSide, j0 = t % nj * kSide;
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
    constexpr int N = Row<T>::kVec, kEach = kSide * kSide / N / 256, kRow = kSide / N;
    float x[kEach][N];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int e = threadIdx.x + 256 * k, r = e / kRow, c = e % kRow * N;
        const T *at = g + (int64_t)(r0 + r) * cols + c0 + c;
        const bool row = r0 + r < rows;
        if (row && c0 + c + N <= cols) Row<T>::unpack(Row<T>::load(at), x[k]);
        else {
#pragma unroll
            for (int u = 0; u < N; ++u) x[k][u] = row && c0 + c + u < cols ? Elem<T>::ld(at + u) : 0.0f;
        }
    }
    __syncthreads();
    const double inv = inv_s;
    // (in 64 bits: 1 / |G| may be beyond f32's range)  Beyond G's rows and columns X is 0 whatever the norm is.
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int e = threadIdx.x + 256 * k, r = e / kRow, c = e % kRow * N;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            x[k][u] = r0 + r < rows && c0 + c + u < cols ? (float)((double)x[k][u] * inv) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < N; u += 4) *(f32x4_t *)(tile + sums_at(r, c + u)) = f32x4_t{x[k][u], x[k][u + 1], x[k][u + 2], x[k][u + 3]};
    }
    __syncthreads();
    const int64_t base = m * (int64_t)o.sp * o.lp + (int64_t)i0 * o.lp + j0;
#pragma unroll 2
    for (int k = 0; k < kSide * kSide / 8 / 256; ++k) {
        const int e = threadIdx.x + 256 * k, r = e >> 4, c = (e & 15) * 8;
        float v[8];
        if (o.transposed) read_down(tile, c, r, v);
        else read_along(tile, r, c, v);
        put8<true>(o.X, base + (int64_t)r * o.lp + c, v);
    }
}

struct Plan {
    int s, l, sp, lp, parts;
    int64_t chunk;             // matrices at a time
    size_t norm, X, Y, A, B, total;
    bool split;
};

Plan plan(int64_t batch, int64_t rows, int64_t cols, int dtype_out) {
    Plan p;
    p.s = (int)(rows < cols ? rows : cols);
    p.l = (int)(rows < cols ? cols : rows);
    p.sp = (p.s + kSide - 1) / kSide * kSide;
    p.lp = (p.l + kSide - 1) / kSide * kSide;
    p.split = dtype_out == R3_F32;
    const int64_t elems = rows * cols;
    p.parts = (int)((elems + kNormElems - 1) / kNormElems);
    if (p.parts > kNormParts) p.parts = kNormParts;
    const size_t x = (size_t)p.sp * p.lp * 4, a = (size_t)p.sp * p.sp * (p.split ? 4 : 2);   // of a matrix: X or Y, A or B
    const size_t most = (size_t)4 << 30;
    const int64_t fit = (int64_t)(most / (2 * (x + a)));
    p.chunk = fit < 1 ? 1 : fit < batch ? fit : batch;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    p.norm = take((size_t)batch * p.parts * sizeof(double));
    p.X = take(x * p.chunk);
    p.Y = take(x * p.chunk);
    p.A = take(a * p.chunk);
    p.B = take(a * p.chunk);
    p.total = o;
    return p;
}

template <int MODE, bool SPLIT, typename OUT> hipError_t tiles(const Ortho &o, int64_t matrices, hipStream_t s) {
    auto k = ortho_tile_kernel<MODE, SPLIT, OUT>;
    (void)hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    k<<<(unsigned)(matrices * o.ntiles), 256, kLdsBytes, s>>>(o);
    return hipGetLastError();
}

template <bool SPLIT, typename OUT> hipError_t iterate(Ortho o, int64_t matrices, int steps, const float *coef, float scale, hipStream_t s) {
    const int ns = o.sp / kSide, half = ns * (ns + 1) / 2, full = ns * (o.lp / kSide);
    const float a = coef[0], b = coef[1], c = coef[2];
    for (int k = 0; k < steps; ++k) {
        // what is taken out of the polynomial and applied to X itself
        const float apart = k >= steps - 2 ? a + b + c : a;
        o.ntiles = half;
        hipError_t e = tiles<kGram, SPLIT, float>(o, matrices, s);
        if (e != hipSuccess) return e;
        o.a = a - apart;
        o.b = b;
        o.c = c;
        e = tiles<kPoly, SPLIT, float>(o, matrices, s);
        if (e != hipSuccess) return e;
        o.ntiles = full;
        o.a = apart;
        o.out = scale / kUnit;
        e = k + 1 < steps ? tiles<kStep, SPLIT, float>(o, matrices, s) : tiles<kLast, SPLIT, OUT>(o, matrices, s);
        if (e != hipSuccess) return e;
        const Pair t = o.X;
        o.X = o.Y;
        o.Y = t;
    }
    return hipSuccess;
}

}  // namespace

size_t orthogonalize_ws_bytes(int64_t batch, int64_t rows, int64_t cols, int dtype_out) { return plan(batch, rows, cols, dtype_out).total; }

// Whether every element stays in (-15, 15): a matrix's are at most its largest singular value, which is at most 1 at the start and then
// what the quintic makes of it.
bool orthogonalize_in_range(int steps, const float *coef) {
    const double a = coef[0], b = coef[1], c = coef[2];
    double r = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double apart = k >= steps - 2 ? a + b + c : a;
        double x_most = 0.0, b_most = 0.0;
        for (int i = 0; i <= 1024; ++i) {
            const double x = r * i / 1024, y = x * x;
            x_most = std::fmax(x_most, std::fabs(x * (a + y * (b + y * c))));
            b_most = std::fmax(b_most, std::fabs(a - apart + y * (b + y * c)));
        }
        const double room = 1.01;    // for roundings and what lies between the points
        if (!(r * r * room < 15.0 && b_most * room < 15.0 && x_most * room < 15.0)) return false;
        r = x_most * 1.001;
    }
    return true;
}

hipError_t launch_orthogonalize(int64_t batch, int64_t rows, int64_t cols, int dtype_in, const void *G, int dtype_out, void *out, int steps,
                                const float *coef, float eps, float scale, int32_t *status, void *ws, hipStream_t s) {
    ProfScope ps(PROF_ORTHO, s);
    const Plan p = plan(batch, rows, cols, dtype_out);
    char *base = (char *)ws;
    double *part = (double *)(base + p.norm);
    const int64_t elems = rows * cols;
    const size_t eb = dtype_in == R3_BF16 ? 2 : 4, ob = dtype_out == R3_BF16 ? 2 : 4;
    for (int64_t m0 = 0; m0 < batch; m0 += p.chunk) {
        const int64_t nm = batch - m0 < p.chunk ? batch - m0 : p.chunk;
        const int64_t xs = (int64_t)p.sp * p.lp * p.chunk, as = (int64_t)p.sp * p.sp * p.chunk;
        Ortho o = {};
        o.s = p.s; o.l = p.l; o.sp = p.sp; o.lp = p.lp;
        o.transposed = rows > cols;
        auto pair = [&](size_t at, int64_t n) { return Pair{(f16_t *)(base + at), (f16_t *)(base + at) + n}; };
        o.X = pair(p.X, xs); o.Y = pair(p.Y, xs); o.A = pair(p.A, as); o.B = pair(p.B, as);
        o.O = (char *)out + (size_t)m0 * elems * ob;
        const char *g = (const char *)G + (size_t)m0 * elems * eb;
        const unsigned ntiles = (unsigned)(nm * (p.sp / kSide) * (p.lp / kSide));
        auto start = [&](auto type) {
            typedef decltype(type) T;
            ortho_norm_kernel<T><<<(unsigned)(nm * p.parts), 256, 0, s>>>((const T *)g, elems, p.parts, part);
            (void)hipFuncSetAttribute((const void *)ortho_start_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
            ortho_start_kernel<T><<<ntiles, 256, kLdsBytes, s>>>((const T *)g, o, p.parts, part, (double)eps, status);
        };
        if (dtype_in == R3_BF16) start(bf16_t{});
        else start(float{});
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        e = p.split ? iterate<true, float>(o, nm, steps, coef, scale, s) : iterate<false, bf16_t>(o, nm, steps, coef, scale, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace r3
