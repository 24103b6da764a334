// Newton-Schulz orthogonalisation (r3_ortho.hip has the mathematics and the numbers' scale) of matrices with a short side of at most 128:
// such a matrix's A = X X^T fits into a compute unit's LDS as a pair of f16, and its X goes by in slabs of 64 columns.
//
// A work-group has a run of a matrix's slabs.  A step of it: A, then B = b A + c A A + .. into LDS; of each slab X' = a X + B X, and at
// once X' X'^T added to its part of the next step's A, in registers.  So a step is one launch that reads and writes X once, and another
// that joins the parts where there are more than a few; as products over tiles it was five, each of which waited for the one before (1 x
// 2048 x 128 f32: 27 launches, 128 us | 10, 75 us; 256 x 128 x 1024: 878 | 353).  Where a work-group has a whole matrix, B is the smaller
// part of its work; where work-groups share one, each makes B for itself, which costs as much as a slab and a half.
//
// Two steps as one (r3_ortho.hip) are four products more of matrices that are in LDS, 12 us, for a pass over X and a join less: everywhere
// for bf16 results (1 x 64 x 2048 54 -> 41 us, 128 x 100 x 700 211 -> 154); for f32 ones at the start alone (256 x 128 x 1024 411 -> 353),
// as later pairs cost exactness (1 x 2048 x 128: 5.1e-6 of the result instead of 1.1e-6; f32 products 1.5e-6).
//
// Bound by latencies where matrices are few (a step of one slab is 10 us, some 2 of them products), by memory where they are many (256 x
// 128 x 1024: 72 us a step, 268 MB, 3.7 TB/s; matrix pipes 39 % busy).
//
// X, A and B are pairs of f16 times 2^12 for results of either type: products are hi hi, hi lo, lo hi.  These matrices have few directions
// in which an error could be lost (3 x 5, f16 operands: 6e-3 of the norm at worst), and the two products more hide behind the rest.
#include <algorithm>

#include "r3_kernels.h"
#include "r3_mfma2.h"
#include "r3_vec.h"

namespace r3 {
namespace {

typedef _Float16 f16_t;
typedef f16_t f16x4_t __attribute__((ext_vector_type(4)));

constexpr float kUnit = 4096.0f;      // what is stored is times this
constexpr int kSlab = 64;             // columns
constexpr int kFew = 2;               // parts of A that a step joins by itself

enum { kStart = 0, kStep = 1, kLast = 2 };
struct Narrow {
    int s, l, slabs, pieces, parts;      // pieces: work-groups of a matrix; parts: of A as it is read
    bool transposed;
    const void *G;
    void *O;
    char *X;                             // [matrix][slab]: SP rows of hi, SP rows of lo, as they are in LDS
    const float *A;                      // [matrix][part]: sums as the threads have them
    float *A_to;
    int norms;                           // of a matrix: parts of |G|^2
    const double *norm;
    double eps;
    bool two;                            // two steps: X'' = apart X + (rest I + a B + a B' + B' B) X, B' = b A' + c A' A', A' = (a + B) (a + B) A
    float apart, rest, a, b, c, out;     // X' = apart X + (rest I + B) X, B = b A + c A A
    int32_t *status;
};

template <int SP> struct Shape {
    static constexpr int kWaves = SP == 128 ? 8 : 4, kThreads = 64 * kWaves;
    static constexpr int kPlane = SP * kSlab * 2, kBytes = 2 * kPlane;           // hi or lo of a slab, both
    static constexpr int kPitch = SP * 2 + 16;                                   // bytes of a row of A or B
    static constexpr int kMatrix = SP * kPitch;                                  // hi or lo of it
    static constexpr int kRoom = 2 * kBytes < 2 * kMatrix ? 2 * kMatrix : 2 * kBytes;     // two slabs, or before them a second matrix
    static constexpr int kLds = 2 * kMatrix + kRoom;
    static constexpr int kGP = SP == 128 ? 4 : 2, kGQ = 2;                       // 16 x 16 tiles of a wave, of A: 64 x 32 or 32 x 32
    static constexpr int64_t kSums = SP * SP;
};
static_assert(Shape<128>::kLds <= 160 * 1024, "");

// A slab in LDS: rows of 128 bytes, the 16-byte chunk c of row r at c ^ ((r >> 1) & 7), so that both ways of reading it (KcFrag16's along
// rows, and down columns) meet few banks twice.
__device__ __forceinline__ int slab_at(int row, int col) { return row * 128 + ((((col >> 3) ^ (row >> 1)) & 7) << 4) + (col & 7) * 2; }
// 32 rows from row 32 kk on of 16 columns, as an operand whose k are rows: two transposing reads of 4 k each
struct DownFrag {
    int at;
    __device__ __forceinline__ void init(int col0) {
        const int lane = lane_id(), i = lane & 15, k = 8 * (lane >> 4) + (i >> 2);
        at = slab_at(k, col0 + 4 * (i & 3));
    }
    __device__ __forceinline__ bf16x8_t read(const char *plane, int kk) const {
        // (rows 32 on have the same swizzle, rows 4 on the other one in bit 1)
        const char *p = plane + kk * (32 * 128) + at, *q = plane + kk * (32 * 128) + ((at + 4 * 128) ^ 32);
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(q));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// 32 k (64 bytes) from k = 32 kk on of 16 rows of A or B
template <int PITCH> __device__ __forceinline__ bf16x8_t row_frag(const char *m, int row0, int kk) {
    const int lane = lane_id();
    return *(const bf16x8_t *)(m + (row0 + (lane & 15)) * PITCH + kk * 64 + (lane >> 4) * 16);
}
// acc += P Q for pairs, the small products apart
__device__ __forceinline__ void pair_mfma(f32x4_t &large, f32x4_t &small, const bf16x8_t (&p)[2], const bf16x8_t (&q)[2]) {
    small = MfmaF16::run(p[1], q[0], small);
    small = MfmaF16::run(p[0], q[1], small);
    large = MfmaF16::run(p[0], q[0], large);
}
// four elements at any address, of which `left` are there
__device__ __forceinline__ f32x4_t load4(const float *p, int left) {
    if (left >= 4) return Row<float>::load(p);
    return f32x4_t{left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, 0.0f};
}
__device__ __forceinline__ f32x4_t load4(const bf16_t *p, int left) {
    typedef uint32_t V __attribute__((ext_vector_type(2)));
    typedef V U __attribute__((aligned(2)));
    if (left >= 4) {
        const V v = *(const U *)p;
        return f32x4_t{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u), __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
    }
    auto one = [&](int u) { return left > u ? Elem<bf16_t>::ld(p + u) : 0.0f; };
    return f32x4_t{one(0), one(1), one(2), 0.0f};
}
__device__ __forceinline__ void store4(float *p, const float *v) { Row<float>::store(p, v); }
__device__ __forceinline__ void store4(bf16_t *p, const float *v) {
    typedef uint32_t V __attribute__((ext_vector_type(2)));
    typedef V U __attribute__((aligned(2)));
    *(U *)p = V{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
// four values as a pair, `lo_off` bytes apart
__device__ __forceinline__ void put_pair(char *at, int lo_off, const float *v) {
    f16x4_t h, lo;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        h[u] = (f16_t)v[u];
        lo[u] = (f16_t)(v[u] - (float)h[u]);
    }
    *(f16x4_t *)at = h;
    *(f16x4_t *)(at + lo_off) = lo;
}

template <int SP, int MODE, typename T> __global__ void __launch_bounds__(Shape<SP>::kThreads, 1) ortho_narrow_kernel(Narrow o) {
    typedef Shape<SP> H;
    constexpr int NT = H::kThreads, kP = H::kGP, kQ = H::kGQ;
    extern __shared__ __align__(1024) char lds[];
    char *const M = lds, *const S = lds + 2 * H::kMatrix;     // A, and what comes of it; two slabs
    const int64_t m = blockIdx.x / o.pieces, elems = (int64_t)o.s * o.l;
    const int piece = (int)(blockIdx.x - m * o.pieces);
    const int j0 = (int)((int64_t)o.slabs * piece / o.pieces), j1 = (int)((int64_t)o.slabs * (piece + 1) / o.pieces);
    char *X = o.X + m * o.slabs * (int64_t)H::kBytes;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, c4 = 4 * (lane >> 4);
    // of A: waves 2 along (p), the others down; of a slab: 2 along by 32 columns, the others down by 32 rows
    const int gp = (wave & 1) * 16 * kP, gq = (wave >> 1) * 16 * kQ, xp = (wave & 1) * 32, xq = (wave >> 1) * 32;

    f32x4_t A[kP][kQ], As[kP][kQ];      // large and small products
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < kP; ++i)
#pragma unroll
            for (int j = 0; j < kQ; ++j) A[i][j] = As[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    };
    // += slab slab^T
    KcFrag16 fp, fq;
    fp.init(gp, lane);
    fq.init(gq, lane);
    auto gram = [&](const char *slab) {
#pragma unroll
        for (int u = 0; u < kSlab / 32; ++u) {
            bf16x8_t p[kP][2], q[kQ][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < kP; ++i) p[i][h] = fp.read(slab + h * H::kPlane, i, u);
#pragma unroll
                for (int j = 0; j < kQ; ++j) q[j][h] = fq.read(slab + h * H::kPlane, j, u);
            }
#pragma unroll
            for (int j = 0; j < kQ; ++j)
#pragma unroll
                for (int i = 0; i < kP; ++i) pair_mfma(A[i][j], As[i][j], p[i], q[j]);
        }
    };
    constexpr int kChunks = H::kBytes / 16 / NT;      // 16-byte pieces of a slab to a thread
    auto load = [&](int j, char *slab) {
        const rsrc_t d = src_rsrc_inside(Src{X + (int64_t)j * H::kBytes, 0, 0}, 0);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) lds_load16(d, lds_addr(slab) + 1024 * (wave + H::kWaves * i), (wave + H::kWaves * i) * 1024 + lane * 16);
    };
    auto store = [&](int j, const char *slab) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int at = (tid + NT * i) * 16;
            *(uint4 *)(X + (int64_t)j * H::kBytes + at) = *(const uint4 *)(slab + at);
        }
    };
    auto sums_of = [&](int64_t part, int i, int j) { return part * H::kSums + (((int64_t)i * kQ + j) * NT + tid) * 4; };

    if constexpr (MODE == kStart) {
        // X = G / (|G| + eps)
        const T *G = (const T *)o.G + m * elems;
        const double sum = wave_sum(lane < o.norms ? o.norm[m * o.norms + lane] : 0.0), n = sqrt(sum) + o.eps;
        // (in 64 bits: 1 / |G| may be beyond f32's range)
        const double inv = n == 0.0 ? 0.0 : isfinite(sum) ? (double)kUnit / n : (double)NAN;
        if (tid == 0 && piece == 0 && !isfinite(sum) && o.status) atomicOr(o.status, R3_DATA_NONFINITE);
        clear();
        // A thread has a block of 4 x 4 of a slab: four loads of four elements along G's rows (a wave: 32 x 32), and eight bytes of four rows
        // to LDS, each bank as often as another.  (Single elements: 256 x 128 x 1024 153 us instead of 60.)
        const int row0 = 32 * (wave % (SP / 32)) + 4 * (lane & 7), col0 = 32 * (wave / (SP / 32)) + 4 * (lane >> 3);
        f32x4_t v[4];
        auto fetch = [&](int j) {
            const int at = o.transposed ? j * kSlab + col0 : row0, along = o.transposed ? row0 : j * kSlab + col0;
            const int lines = o.transposed ? o.l : o.s, width = o.transposed ? o.s : o.l;
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = at + u < lines ? load4(G + (int64_t)(at + u) * width + along, width - along) : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        };
        fetch(j0);
        for (int j = j0; j < j1; ++j) {
            char *slab = S + (j & 1) * H::kBytes;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)      // (beyond G's rows and columns X is 0 whatever the norm is)
                    x[u] = row0 + i < o.s && j * kSlab + col0 + u < o.l ? (float)((double)(o.transposed ? v[u][i] : v[i][u]) * inv) : 0.0f;
                put_pair(slab + slab_at(row0 + i, col0), H::kPlane, x);
            }
            // (two slabs: everybody has left the one before the last)
            __syncthreads();
            if (j + 1 < j1) fetch(j + 1);
            gram(slab);
            store(j, slab);
        }
    } else {
        if (!o.two) load(j0, S + (j0 & 1) * H::kBytes);
#pragma unroll
        for (int i = 0; i < kP; ++i)
#pragma unroll
            for (int j = 0; j < kQ; ++j) A[i][j] = *(const f32x4_t *)(o.A + sums_of(m * o.parts, i, j));
        for (int k = 1; k < o.parts; ++k)
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) A[i][j] += *(const f32x4_t *)(o.A + sums_of(m * o.parts + k, i, j));
        // a matrix to LDS; everybody has read what was there
        auto put = [&](char *to, const f32x4_t (&v)[kP][kQ]) {
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) {
                    float x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[u] = v[i][j][u];
                    put_pair(to + (gq + 16 * j + r) * H::kPitch + (gp + 16 * i + c4) * 2, H::kMatrix, x);
                }
        };
        // v = x v + y P Q, of matrices in LDS that commute; everybody meets
        auto product = [&](f32x4_t (&v)[kP][kQ], float x, float y, const char *P, const char *Q) {
            f32x4_t large[kP][kQ], small[kP][kQ];
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) large[i][j] = small[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            __syncthreads();
#pragma unroll
            for (int kk = 0; kk < SP / 32; ++kk) {
                bf16x8_t p[kP][2], q[kQ][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int i = 0; i < kP; ++i) p[i][h] = row_frag<H::kPitch>(P + h * H::kMatrix, gp + 16 * i, kk);
#pragma unroll
                    for (int j = 0; j < kQ; ++j) q[j][h] = row_frag<H::kPitch>(Q + h * H::kMatrix, gq + 16 * j, kk);
                }
#pragma unroll
                for (int j = 0; j < kQ; ++j)
#pragma unroll
                    for (int i = 0; i < kP; ++i) pair_mfma(large[i][j], small[i][j], p[i], q[j]);
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) {
                    const f32x4_t s = (large[i][j] + small[i][j]) * (y * (1.0f / kUnit));
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[i][j][u] = fmaf(x, v[i][j][u], s[u]);
                }
        };
        put(M, A);
        if (o.two) {
            f32x4_t B[kP][kQ];
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) B[i][j] = A[i][j];
            product(B, o.b, o.c, M, M);       // B
            put(S, B);
            product(A, o.a, 1.0f, M, S);      // (a + B) A
            put(M, A);
            product(A, o.a, 1.0f, M, S);      // A'
            put(M, A);
            product(A, o.b, o.c, M, M);       // B'
            put(M, A);
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) A[i][j] += B[i][j];
            product(A, o.a, 1.0f, M, S);
            load(j0, S + (j0 & 1) * H::kBytes);
        } else product(A, o.b, o.c, M, M);
#pragma unroll
        for (int i = 0; i < kP; ++i)
#pragma unroll
            for (int j = 0; j < kQ; ++j)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (gq + 16 * j + r == gp + 16 * i + c4 + u && gq + 16 * j + r < o.s) A[i][j][u] += o.rest * kUnit;
        put(M, A);
        if constexpr (MODE == kStep) clear();
        DownFrag down[2];
        down[0].init(xp);
        down[1].init(xp + 16);
        for (int j = j0; j < j1; ++j) {
            char *slab = S + (j & 1) * H::kBytes;
            asm volatile("" ::: "memory");
            window_barrier<0>();      // the slab has come, B is there, everybody has left the slab before
            asm volatile("" ::: "memory");
            if (j + 1 < j1) load(j + 1, S + ((j + 1) & 1) * H::kBytes);
            f32x4_t x[2][2], xs[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) x[i][k] = xs[i][k] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < SP / 32; ++kk) {
                bf16x8_t p[2][2], q[2][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        p[i][h] = down[i].read(slab + h * H::kPlane, kk);
                        q[i][h] = row_frag<H::kPitch>(M + h * H::kMatrix, xq + 16 * i, kk);
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) pair_mfma(x[i][k], xs[i][k], p[i], q[k]);
            }
            // a lane's: rows xq + 16 k + r, columns xp + 16 i + c4 .. + 3
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const char *at = slab + slab_at(xq + 16 * k + r, xp + 16 * i + c4);
                    const f16x4_t h = *(const f16x4_t *)at, lo = *(const f16x4_t *)(at + H::kPlane);
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[i][k][u] = fmaf(o.apart, (float)h[u] + (float)lo[u], (x[i][k][u] + xs[i][k][u]) * (1.0f / kUnit));
                }
            if constexpr (MODE == kLast) {
                T *O = (T *)o.O + m * elems;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int row = xq + 16 * k + r, col = j * kSlab + xp + 16 * i + c4;
                        float v[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) v[u] = x[i][k][u] * o.out;
                        if (row >= o.s) continue;
                        if (!o.transposed && col + 4 <= o.l) store4(O + (int64_t)row * o.l + col, v);
                        else {
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                if (col + u < o.l) Elem<T>::st(O + (o.transposed ? (int64_t)(col + u) * o.s + row : (int64_t)row * o.l + col + u), v[u]);
                        }
                    }
            } else {
                // Everybody has read the slab: X' in its place.  (Bare waits, so that the next slab's loads stay on their way.)
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float v[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) v[u] = x[i][k][u];
                        put_pair(slab + slab_at(xq + 16 * k + r, xp + 16 * i + c4), H::kPlane, v);
                    }
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                gram(slab);
                store(j, slab);
            }
        }
    }
    if constexpr (MODE != kLast) {
#pragma unroll
        for (int i = 0; i < kP; ++i)
#pragma unroll
            for (int j = 0; j < kQ; ++j) *(f32x4_t *)(o.A_to + sums_of(m * o.pieces + piece, i, j)) = (A[i][j] + As[i][j]) * (1.0f / kUnit);
    }
}

// the parts of a matrix's A, in their order
__global__ void __launch_bounds__(64) ortho_narrow_join_kernel(const float *__restrict__ parts, int pieces, int64_t sums, float *__restrict__ A) {
    const int per = (int)(sums / 256);
    const int64_t m = blockIdx.x / per, at = (int64_t)(blockIdx.x - m * per) * 256 + threadIdx.x * 4;
    const float *from = parts + m * pieces * sums + at;
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 16
    for (int k = 0; k < pieces; ++k) sum += *(const f32x4_t *)(from + k * sums);
    *(f32x4_t *)(A + m * sums + at) = sum;
}

struct Plan {
    int slabs, pieces;
    int64_t chunk;             // matrices at a time
    size_t X, A, A2, total;
};
template <int SP> Plan plan(int64_t batch, int64_t l) {
    typedef Shape<SP> H;
    Plan p;
    p.slabs = (int)((l + kSlab - 1) / kSlab);
    const size_t x = (size_t)p.slabs * H::kBytes;
    p.chunk = std::min<int64_t>(batch, std::max<int64_t>(1, (int64_t)(((size_t)4 << 30) / (x + 4 * H::kSums * sizeof(float)))));
    // Work-groups to a matrix: the fewest rounds of slabs over the card, where B costs as much as one and a half (3.2 us a slab of 128
    // rows, 1.5 us of 64), a launch that joins A as much as three, and a part of A that is written and read a share of the card's
    // bandwidth.  (us a call, with 32 | 16 | 8 work-groups: 1 x 128 x 2048 f32 78 | 90 | 129, 8 x 141 | 119 | 142, 16 x 194 | 135 | 152;
    // with 4 | 2 | 1: 64 x 128 x 768 154 | 166 | 242, 128 x 276 | 201 | 255, 200 x 470 | 340 | 274, 128 x 64 x 1024 130 | 126 | 180.)
    p.pieces = 1;
    double best = 0.0;
    for (int n = 1; n <= std::min(p.slabs, 256); ++n) {
        const int64_t rounds = (p.chunk * n + 255) / 256;
        const double cost = (double)rounds * ((p.slabs + n - 1) / n + 1.5) + (n > kFew ? 3.0 : 0.3 * n) + (n > 1 ? 0.012 * SP / 128 * p.chunk * n : 0.0);
        if (n == 1 || cost < best) {
            best = cost;
            p.pieces = n;
        }
    }
    const size_t a = (size_t)p.chunk * H::kSums * sizeof(float);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    p.X = take(x * p.chunk);
    p.A = take(a * p.pieces);
    p.A2 = take(p.pieces > kFew ? a : a * p.pieces);
    p.total = o;
    return p;
}

template <int SP, typename IN, typename OUT> hipError_t run(const NarrowCall &c, hipStream_t s) {
    typedef Shape<SP> H;
    const Plan p = plan<SP>(c.batch, c.l);
    char *base = (char *)c.ws;
    const int64_t elems = (int64_t)c.s * c.l;
    Narrow o = {};
    o.s = c.s; o.l = c.l; o.slabs = p.slabs; o.pieces = p.pieces;
    o.transposed = c.transposed;
    o.X = base + p.X;
    o.norms = c.norms;
    o.eps = c.eps;
    o.out = c.scale / kUnit;
    o.status = c.status;
    o.a = c.coef[0];
    o.b = c.coef[1];
    o.c = c.coef[2];
    hipError_t e = hipSuccess;
    for (int64_t m0 = 0; m0 < c.batch; m0 += p.chunk) {
        const int64_t nm = std::min(p.chunk, c.batch - m0);
        o.G = (const IN *)c.G + m0 * elems;
        o.O = (OUT *)c.O + m0 * elems;
        o.norm = c.norm + m0 * c.norms;
        float *now = (float *)(base + p.A), *other = (float *)(base + p.A2);
        auto go = [&](auto kernel) {
            if (e != hipSuccess) return;
            (void)hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, H::kLds);
            kernel<<<(unsigned)(nm * p.pieces), H::kThreads, H::kLds, s>>>(o);
            e = hipGetLastError();
        };
        // `now`: the work-groups' sums; with many of them `other` is what they are joined into
        o.A_to = now;
        go(ortho_narrow_kernel<SP, kStart, IN>);
        for (int k = 0; k < c.steps && e == hipSuccess;) {
            o.two = c.pairs && ortho_together(k, c.steps, std::is_same<OUT, bf16_t>::value);
            const double apart = ortho_apart(k, c.steps, c.coef) * (o.two ? ortho_apart(k + 1, c.steps, c.coef) : 1.0);
            o.apart = (float)apart;
            o.rest = (float)((double)o.a * (o.two ? o.a : 1.0) - apart);
            k += o.two ? 2 : 1;
            o.parts = p.pieces;
            o.A = now;
            if (p.pieces > kFew) {
                ortho_narrow_join_kernel<<<(unsigned)(nm * (H::kSums / 256)), 64, 0, s>>>(now, p.pieces, H::kSums, other);
                e = hipGetLastError();
                o.parts = 1;
                o.A = other;
            } else std::swap(now, other);
            o.A_to = now;
            if (k < c.steps) go(ortho_narrow_kernel<SP, kStep, float>);
            else go(ortho_narrow_kernel<SP, kLast, OUT>);
        }
        if (e != hipSuccess) return e;
    }
    return e;
}

}  // namespace

size_t ortho_narrow_ws_bytes(int64_t batch, int64_t s, int64_t l) { return (s <= 64 ? plan<64>(batch, l) : plan<128>(batch, l)).total; }

hipError_t launch_ortho_narrow(const NarrowCall &c, int dtype_in, int dtype_out, hipStream_t s) {
    auto by_out = [&](auto sp, auto in) {
        constexpr int SP = decltype(sp)::value;
        typedef decltype(in) IN;
        return dtype_out == R3_BF16 ? run<SP, IN, bf16_t>(c, s) : run<SP, IN, float>(c, s);
    };
    auto by_in = [&](auto sp) { return dtype_in == R3_BF16 ? by_out(sp, bf16_t{}) : by_out(sp, float{}); };
    return c.s <= 64 ? by_in(std::integral_constant<int, 64>{}) : by_in(std::integral_constant<int, 128>{});
}

}  // namespace r3
