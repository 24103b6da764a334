// Log-probabilities of given tokens, entropy and the most probable alternatives of a row of logits, and the gradient:
//   x_v = s (z_v - m), m = max z;  S = sum e^x;  log p_v = x_v - log S;  H = log S - (sum e^x x) / S
//   dz_v = s ([v = t] dlogp - p_v (dlogp + dH (log p_v + H)))
// Both read the logits once (and the gradient writes once): HBM-bound.
#include <algorithm>
#include <cfloat>

#include "r3_kernels.h"
#include "r3_vec.h"

namespace r3 {
namespace {

constexpr int kMaxTop = R3_MAX_TOP;
constexpr int kMaxSplit = 64;       // parts of a row: one lane each when they are joined
constexpr float kFar = 1e4f;        // 2^-kFar is 0: exponents are kept above -kFar, so that 0 x (-inf) never arises
constexpr int64_t kRowsAtOnce = 1 << 22;   // work-groups of a launch: a grid has less than 2^32 threads
constexpr float kSpan = 8.0f;       // in powers of two
constexpr float kMostRef = 16777216.0f;   // 2^24
constexpr float kLn2 = 0.693147180559945309f;

// The larger of two numbers; NaN if one is NaN (v_maximum3_f32), so that a row's maximum says whether it holds one.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_max_nan(float v) {
    return over_wave(v, -INFINITY, [](float a, float b) { return max_nan(a, b); });
}

// Running statistics over some of a row's elements: m their maximum, s = sum 2^x, q = sum 2^x x with x = c z - r,
// c = scale log2(e).  The sums refer to a logit b that was the maximum when it was taken, r = c b, and stay with it until a
// logit exceeds `most` = b + kSpan / c: one fused multiply-add to an exponent, with the one rounding, and hardly a change of
// reference in the loop.  q loses what cancels when it is referred to the row's maximum in the end: at most kSpan times the
// rounding of s, and the sums of a piece are made apart, so that few roundings are that large (16384 x 151936, entropies off by
// at most: kSpan = 64, one chain 4e-6 of their size, 64 4e-7, 8 2e-7, 0 2e-7; the time is the same within 1 %).
//
// r carries the rounding of c b into every exponent, and out again in the end: half a unit in c b's last place, 1/2 at kMostRef,
// but past a float's largest exponent from 2^32 on.  Where |c b| is above kMostRef (mask values like -1e9 are), or there is
// nothing but -inf so far, most = -inf, r = b and x = c (z - b) (4096 x 151936 bf16 with the first half at -1e9 183 us, random
// halves 183; at -inf 187 and 188).
//
// Elements come in pieces: `where` is the piece that holds m, m2 the largest of the other pieces.  `masked`: a piece has held
// -inf.
struct Stat {
    float m, s, q, r, most, m2;
    int where;
    bool masked;
};
__device__ __forceinline__ Stat no_stat() { return {-INFINITY, 0.0f, 0.0f, -INFINITY, -INFINITY, -INFINITY, 0, false}; }
// a piece's name: its first vector, and whether it is two vectors (NT apart), one, or one of the loose elements
enum { kPair = 0, kOne = 1, kLoose = 2 };
// s and q for exponents less by d
template <bool ENT> __device__ __forceinline__ void shift(Stat &a, float d) {
    const float f = __builtin_amdgcn_exp2f(d);
    if constexpr (ENT) a.q = fmaf(a.s, d, a.q) * f;
    a.s *= f;
}
// s and q for x = c (z - m) instead; m is at least the reference (or NaN)
template <bool ENT> __device__ __forceinline__ void refer_to(Stat &a, float m, float c) {
    shift<ENT>(a, fmaxf(a.most > -INFINITY ? fmaf(-m, c, a.r) : (a.r - m) * c, -kFar));   // (-inf less -inf: -kFar)
}

// N more elements, a piece of the name given.
template <bool ENT, bool TOP, int N>
__device__ __forceinline__ void take(Stat &a, const float (&z)[N], float c, float span, int name) {
    float hi = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) hi = max_nan(hi, z[i]);
    if constexpr (TOP) {
        a.m2 = __builtin_amdgcn_fmed3f(a.m, hi, a.m2);
        a.where = hi > a.m ? name : a.where;
    }
    a.m = max_nan(a.m, hi);
    if (!(hi <= a.most)) {   // the first ones, a much larger one, a NaN
        refer_to<ENT>(a, a.m, c);
        const float r = a.m * c;
        const bool moderate = fabsf(r) <= kMostRef;
        a.most = moderate ? a.m + span : -INFINITY;
        a.r = moderate ? r : a.m;
        if (moderate) shift<ENT>(a, fmaf(a.m, c, -a.r));   // from x = c (z - b) to x = c z - r
    }
    if (a.most > -INFINITY) {
        // A wave that has met masked logits goes on with guarded exponents: where some are masked, more are (4096 x 151936
        // bf16, half of it masked, 227 -> 198 us; 188 unmasked).  Not beside the search for alternatives, where the test
        // costs unmasked rows as much as it gives masked ones (200 -> 209, 240 -> 215).
        if (TOP || !__any(a.masked)) {
            float s = 0.0f, q = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = fmaf(z[i], c, -a.r), e = __builtin_amdgcn_exp2f(x);
                s += e;
                if constexpr (ENT) q = fmaf(e, x, q);
            }
            if (!ENT || q == q) {   // (an x of -inf makes q a NaN)
                a.s += s;
                a.q += q;
                return;
            }
            a.masked = true;
        }
        float s = 0.0f, q = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float x = fmaxf(fmaf(z[i], c, -a.r), -kFar), e = __builtin_amdgcn_exp2f(x);
            s += e;
            q = fmaf(e, x, q);
        }
        a.s += s;
        a.q += q;
        return;
    }
    float s = 0.0f, q = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = fmaxf((z[i] - a.r) * c, -kFar), e = __builtin_amdgcn_exp2f(x);
        s += e;
        if constexpr (ENT) q = fmaf(e, x, q);
    }
    a.s += s;
    a.q += q;
}

// What is kept of a part of a row: maximum and sums for x = c (z - m).
struct Part {
    float m, s, q;
};

// A logit and its place in one whole number: larger logits first, then lower places.  0: none.
typedef unsigned long long key_t;
__device__ __forceinline__ uint32_t order_of(float z) {   // of finite numbers and infinities
    const uint32_t b = __float_as_uint(z + 0.0f);         // -0 equals +0
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ key_t make_key(float z, int v) { return ((key_t)order_of(z) << 32) | (0xffffffffu - (uint32_t)v); }
__device__ __forceinline__ float key_logit(key_t k) { return of_order((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_place(key_t k) { return (int)(0xffffffffu - (uint32_t)k); }

struct Args {
    int64_t n, ld, row0;            // rows row0 .. n - 1
    int V, top, nsplit, seg;        // seg: elements of one part of a row
    float scale, c, span;           // c = scale log2(e), span = kSpan / c
    const void *logits;
    const int32_t *target;
    float *logp, *entropy, *stats, *top_logp;
    int32_t *top_id, *status;
    Part *part;                     // [n][nsplit], and
    key_t *part_keys;               // [n][nsplit][top], where rows are cut
};

// scale (z - m), of halves: z - m itself may be past the range where scale < 1
__device__ __forceinline__ float log_odds(float z, float m, float scale) {
    const float d = (0.5f * z - 0.5f * m) * scale;
    return d + d;
}

// The largest term of s is 1, whatever rounding says: no log-probability is above 0, no entropy (below) under it.  A sum that is
// a NaN stays one (fmaxf would make it 1).
__device__ __forceinline__ void settle(Part &r) {
    if (r.m > -INFINITY) r.s = r.s < 1.0f ? 1.0f : r.s;
}

// What a row comes to, by the thread that has it; ls = log r.s.
__device__ __forceinline__ void put_row(const Args &a, int64_t row, const Part &r, float ls, float zt) {
    const float nan = __uint_as_float(0x7fc00000u);
    const bool bad = !(r.m < INFINITY), none = r.m == -INFINITY;
    if (bad && a.status) atomicOr(a.status, R3_DATA_NONFINITE);
    if (a.logp) a.logp[row] = bad ? nan : none ? -INFINITY : log_odds(zt, r.m, a.scale) - ls;
    if (a.entropy) {
        const float h = ls - r.q * kLn2 / r.s;
        a.entropy[row] = bad ? nan : none || h < 0.0f ? 0.0f : h;
    }
    if (a.stats) {
        a.stats[2 * row] = bad ? nan : r.m;
        a.stats[2 * row + 1] = bad ? nan : r.s;
    }
}
__device__ __forceinline__ void put_top(const Args &a, int64_t row, int rank, key_t k, float m, float ls) {
    a.top_logp[row * a.top + rank] = k ? log_odds(key_logit(k), m, a.scale) - ls : -INFINITY;
    a.top_id[row * a.top + rank] = k ? key_place(k) : -1;
}
// A row that is left out (by its target) or has no alternatives.
__device__ __forceinline__ void put_no_top(const Args &a, int64_t row, int tid, float v) {
    if (tid < a.top) {
        a.top_logp[row * a.top + tid] = v;
        a.top_id[row * a.top + tid] = -1;
    }
}
__device__ __forceinline__ void put_left_out(const Args &a, int64_t row, int t, int tid) {
    if (tid == 0) {
        if (t != -1 && a.status) atomicOr(a.status, R3_DATA_IDX_RANGE);
        if (a.logp) a.logp[row] = 0.0f;
        if (a.entropy) a.entropy[row] = 0.0f;
        if (a.stats) a.stats[2 * row] = a.stats[2 * row + 1] = 0.0f;
    }
    put_no_top(a, row, tid, -INFINITY);
}

// How many of the count keys of buf (room for kBuf) are above k: eight reads in flight.
template <int kBuf> __device__ __forceinline__ int rank_of(const key_t *buf, int count, key_t k) {
    int rank = 0;
    for (int q = 0; q < count; q += 8) {
        key_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = buf[min(q + u, kBuf - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += q + u < count && v[u] > k;
    }
    return rank;
}
// Of the candidates in buf[0..count) the `top` largest, each to its rank; keys are distinct (0 is none).  NT / 64
// neighbouring lanes share a candidate's comparisons.
template <int NT, int kBuf, class F> __device__ __forceinline__ void rank_out(const key_t *buf, int count, int top, int tid, F put) {
    constexpr int P = NT / kWave;
    if (P == 1 && count <= kWave) {   // a key to a lane (32000 rows of 1000 with 20 alternatives 41.8 -> 39.3 us)
        const key_t k = tid < count ? buf[tid] : 0;
        const int lo = (int)k, hi = (int)(k >> 32);
        int rank = 0;
        for (int q = 0; q < count; ++q) {
            const key_t other = (key_t)(uint32_t)__builtin_amdgcn_readlane(hi, q) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, q);
            rank += other > k;
        }
        if (tid < count && rank < top) put(rank, k);
        if (tid >= count && tid < top) put(tid, (key_t)0);
        return;
    }
    const int share = tid % P;
    for (int i = tid / P; i < count; i += kWave) {
        const key_t k = buf[i];
        int rank = 0;
        for (int q = share; q < count; q += 4 * P) {
            key_t v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = buf[min(q + u * P, kBuf - 1)];
#pragma unroll
            for (int u = 0; u < 4; ++u) rank += q + u * P < count && v[u] > k;
        }
#pragma unroll
        for (int o = 1; o < P; o <<= 1) rank += __shfl_xor(rank, o, kWave);
        if (share == 0 && rank < top) put(rank, k);
    }
    for (int i = count + tid; i < top; i += NT) put(i, (key_t)0);
}

// A number that at least k of the lanes' values reach, and all but the last bits of the largest such: the upper 16 bits of
// the values' order (what a bf16 has), one at a time by counting lanes.  -inf where fewer than k lanes have more.
__device__ __forceinline__ float reached_by(float v, int k) {
    const uint32_t o = order_of(v);
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t c = t | 1u << bit;
        t = __popcll(__ballot(o >= c)) >= k ? c : t;
    }
    return t <= order_of(-INFINITY) ? -INFINITY : of_order(t);
}

// NT threads to a row (or to one of a.nsplit parts of it); NT = 64: four rows to a work-group, nothing shared between its
// waves.
//
// Alternatives: a thread knows the maximum of its own elements anyway.  The 64 maxima over the threads of one lane number
// are 64 elements of the row, so the k-th largest of them has k elements at or above it: a bound from below for the k-th
// largest element, met by some 64 ln(64 / (64 - k)) elements of a row in random order (24 for k = 20).  A thread whose maximum
// reaches it has that piece read again, and all of its elements if another of its pieces reaches it too (all elements of all such
// threads, a line of memory each, made 4096 x 151936 with 20 alternatives 204 us instead of 159).  Rows that keep more
// candidates than fit (many equal values) are gone through once more in order with the k-th best so far as the bound.
//
// Bound by HBM: 16384 x 151936 bf16 725 us, 6.9 TB/s where a kernel that only reads reaches 7.1 (non-temporal loads; ordinary
// ones 6.3), with the vector pipe about three quarters busy: 8.5 issue slots an element, four of them the exponential.  With
// the maximum as the reference of every sum, as it changes, and guarded exponents it was 11 slots and 825 us.
// Threads to a row: 64 up to 4096 logits (32768 x 4000 bf16 50 us, x 1000 19), 256 up to 64 KB a row, 128 KB with alternatives, whose
// search keeps the others waiting (256 | 512: 4096 x 50257 bf16 71 | 67 us, with 20 alternatives 77 | 85; 8192 x 32000 86 | 89;
// 16384 x 10000 56 | 88), 512 beyond (1024: 4096 x 151936 with alternatives 232 us | 159).  Up to 256 rows that are not cut have a
// compute unit each: 512 threads from 16 KB on, 1024 from 64 KB (200 rows with 8 alternatives, before | so: 32000 bf16 10.1 | 8.7 us,
// f32 13.4 | 10.0, 50257 bf16 12.6 | 9.4, f32 13.5 | 11.8).  Loads on their way: four a thread,
// two where alternatives need the registers (4 | 2: 256 x 151936 with 20 28.4 us | 24.9).
template <typename T, int NT, bool ENT, bool TOP>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT)
token_logprobs_kernel(Args a) {
    typedef Row<T> R;
    constexpr int N = R::kVec, U = TOP ? 2 : 4, W = NT / kWave, kRows = NT == kWave ? 4 : 1;
    constexpr int kBuf = 2 * NT;   // room for the k best and one more element from every thread
    static_assert(kBuf >= NT + kMaxTop, "");
    __shared__ float max_s[kRows][W][kWave], sum_s[kRows][2][W];
    __shared__ int count_s[kRows][3];
    __shared__ int sel_s[TOP ? kRows : 1][TOP ? NT : 1];
    __shared__ key_t buf_s[TOP ? kRows : 1][TOP ? kBuf : 1];
    const int lane = lane_id(), slot = kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0;
    const int tid = kRows > 1 ? lane : (int)threadIdx.x, w = tid / kWave;
    auto sync = [] {
        if constexpr (W > 1) __syncthreads();
        else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    const uint32_t nth = blockIdx.x * kRows + slot, nth_row = a.nsplit == 1 ? nth : nth / (uint32_t)a.nsplit;
    const int split = nth - nth_row * a.nsplit;
    const int64_t row = a.row0 + nth_row, item = row * a.nsplit + split;
    if (row >= a.n) return;
    const int t = a.target ? a.target[row] : 0;
    // Short rows and few long ones wait for latencies: there the target is not waited for, and a row left out is found to
    // be one at the end (32768 x 1000 27 -> 20 us).
    const bool left_out = t < 0 || t >= a.V, late = W == 1 || a.nsplit > 1;
    if (left_out && !late) {
        put_left_out(a, row, t, tid);
        return;
    }
    const T *z = (const T *)a.logits + row * a.ld;
    const int lo = split * a.seg, len = min(a.seg, a.V - lo);
    // elements before the first whole vector at a 16-byte address and behind the last one: a thread each
    const T *zp = z + lo;
    const int head = min(len, (int)((0 - (uintptr_t)zp) % 16 / sizeof(T))), nvec = (len - head) / N, rest = head + nvec * N;
    const int nloose = head + len - rest;
    const T *zv = zp + head;
    auto loose = [&](int i) { return i < head ? i : rest + i - head; };
    if (tid == 0) count_s[slot][0] = count_s[slot][1] = count_s[slot][2] = 0;
    Stat run = no_stat();
    int j = tid;
    typename R::V kept[2];   // a short row's (or part's) vectors stay with their threads
    const bool brief = TOP && nvec <= 2 * NT;
    if (brief) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (j + u * NT < nvec) kept[u] = R::load_once(zv + (int64_t)(j + u * NT) * N);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (j + u * NT < nvec) {
                float f[N];
                R::unpack(kept[u], f);
                take<ENT, TOP>(run, f, a.c, a.span, 0);
            }
        j = nvec;
    }
    // U loads of a thread on their way, consumed two at a time and replaced at once
    if (j + (U - 1) * NT < nvec) {
        typename R::V v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = R::load_once(zv + (int64_t)(j + u * NT) * N);
        for (; j + (2 * U - 1) * NT < nvec; j += U * NT) {
#pragma unroll
            for (int u = 0; u < U; u += 2) {
                float f[2 * N];
                R::unpack(v[u], f);
                R::unpack(v[u + 1], f + N);
                v[u] = R::load_once(zv + (int64_t)(j + (u + U) * NT) * N);
                v[u + 1] = R::load_once(zv + (int64_t)(j + (u + 1 + U) * NT) * N);
                take<ENT, TOP>(run, f, a.c, a.span, 4 * (j + u * NT) + kPair);
            }
        }
#pragma unroll
        for (int u = 0; u < U; u += 2) {
            float f[2 * N];
            R::unpack(v[u], f);
            R::unpack(v[u + 1], f + N);
            take<ENT, TOP>(run, f, a.c, a.span, 4 * (j + u * NT) + kPair);
        }
        j += U * NT;
    }
    for (; j < nvec; j += 2 * NT) {   // what is left, two loads at once (32000 x 1000 18.4 -> 17.2 us)
        typename R::V v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (j + u * NT < nvec) v[u] = R::load_once(zv + (int64_t)(j + u * NT) * N);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (j + u * NT < nvec) {
                float f[N];
                R::unpack(v[u], f);
                take<ENT, TOP>(run, f, a.c, a.span, 4 * (j + u * NT) + kOne);
            }
    }
    float odd = -INFINITY;
    if (tid < nloose) {
        odd = Elem<T>::ld(zp + loose(tid));
        const float f[1] = {odd};
        take<ENT, TOP>(run, f, a.c, a.span, 4 * tid + kLoose);
    }

    float zt = 0.0f;
    if (tid == 0 && !left_out) zt = Elem<T>::ld(z + t);

    const float mine = run.m;
    float top64 = mine;   // the largest of the threads with this lane's number
    if constexpr (W > 1) {
        max_s[slot][w][lane] = mine;
        sync();
#pragma unroll
        for (int i = 0; i < W; ++i) top64 = max_nan(top64, max_s[slot][i][lane]);
    } else if constexpr (TOP) {
        sync();
    }
    const float m = wave_max_nan(top64);
    const bool search = TOP && m > -INFINITY && m < INFINITY;   // (the same in every thread)
    float thr = 0.0f;
    int *sel = sel_s[TOP ? slot : 0];
    key_t *buf = buf_s[TOP ? slot : 0];
    if (search) {
        thr = fmaxf(reached_by(top64, a.top), -FLT_MAX);   // (-inf is never a candidate)
        if (!brief && mine >= thr) {   // from below: threads read as a whole; from above: those of one piece
            if (run.m2 >= thr) sel[atomicAdd(&count_s[slot][0], 1)] = tid;
            else sel[NT - 1 - atomicAdd(&count_s[slot][2], 1)] = run.where;
        }
    }
    refer_to<ENT>(run, m, a.c);
    Part st = {m, wave_total(run.s), ENT ? wave_total(run.q) : 0.0f};
    if constexpr (W > 1) {
        if (lane == 0) {
            sum_s[slot][0][w] = st.s;
            sum_s[slot][1][w] = st.q;
        }
    }
    if constexpr (W > 1 || TOP) sync();
    if constexpr (W > 1) {
        st.s = st.q = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            st.s += sum_s[slot][0][i];
            st.q += sum_s[slot][1][i];
        }
    }
    if (W == 1 && left_out) {
        put_left_out(a, row, t, tid);
        return;
    }
    if (a.nsplit == 1) settle(st);
    const float ls = logf(st.s);
    if (tid == 0) {
        if (a.nsplit == 1) put_row(a, row, st, ls, zt);
        else a.part[item] = st;
    }
    if constexpr (TOP) {
        auto put = [&](int rank, key_t k) {
            if (a.nsplit == 1) put_top(a, row, rank, k, m, ls);
            else a.part_keys[item * a.top + rank] = k;
        };
        if (!search) {
            if (a.nsplit == 1) put_no_top(a, row, tid, m == -INFINITY ? -INFINITY : __uint_as_float(0x7fc00000u));
            else if (tid < a.top) a.part_keys[item * a.top + tid] = 0;
            return;
        }
        const int nsel = count_s[slot][0], none = count_s[slot][2];
        // an element that reaches the bound is a candidate (few are: compacting a wave's with ballots costs more than their atomics,
        // 64 x 151936 with 32 alternatives 19.6 us | 14.8)
        auto offer = [&](float x, int place) {
            if (x >= thr) {
                const int at = atomicAdd(&count_s[slot][1], 1);
                if (at < kBuf) buf[at] = make_key(x, lo + place);
            }
        };
        if (brief && mine >= thr) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (tid + h * NT < nvec) {
                    float f[N];
                    R::unpack(kept[h], f);
#pragma unroll
                    for (int u = 0; u < N; ++u) offer(f[u], head + (tid + h * NT) * N + u);
                }
            if (tid < nloose) offer(odd, loose(tid));
        }
        // the pieces' vectors and all of the other threads', dealt to all threads, two in flight
        const int per = (nvec + NT - 1) / NT, all = 2 * none + nsel * per;
        auto vector_of = [&](int p) {   // (nvec: none)
            if (p >= all) return nvec;
            if (p < 2 * none) {
                const int name = sel[NT - 1 - p / 2], second = p & 1, kind = name & 3;
                return kind == kLoose || (second && kind == kOne) ? nvec : name / 4 + second * NT;
            }
            p -= 2 * none;
            return min(nvec, sel[p / per] + p % per * NT);
        };
        for (int i = tid; i < all; i += 2 * NT) {
            const int q[2] = {vector_of(i), vector_of(i + NT)};
            typename R::V v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (q[h] < nvec) v[h] = R::load(zv + (int64_t)q[h] * N);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (q[h] < nvec) {
                    float f[N];
                    R::unpack(v[h], f);
#pragma unroll
                    for (int u = 0; u < N; ++u) offer(f[u], head + q[h] * N + u);
                }
        }
        for (int i = tid; i < none; i += NT)
            if (const int name = sel[NT - 1 - i]; (name & 3) == kLoose) offer(Elem<T>::ld(zp + loose(name / 4)), loose(name / 4));
        for (int i = tid; i < nsel; i += NT)
            if (sel[i] < nloose) offer(Elem<T>::ld(zp + loose(sel[i])), loose(sel[i]));
        sync();
        int count = count_s[slot][1];
        if (count > kBuf) {
            sync();
            if (tid == 0) count_s[slot][1] = 0;
            sync();
            key_t bound = 0;
            for (int at = 0; at < len; at += NT) {
                const float x = at + tid < len ? Elem<T>::ld(zp + at + tid) : -INFINITY;
                const key_t k = x > -INFINITY ? make_key(x, lo + at + tid) : 0;
                if (k > bound) buf[atomicAdd(&count_s[slot][1], 1)] = k;
                sync();
                count = count_s[slot][1];
                sync();
                if (count > kBuf - NT) {   // keep the best a.top
                    key_t best[kBuf / NT];
                    int rank[kBuf / NT];
#pragma unroll
                    for (int u = 0; u < kBuf / NT; ++u) {
                        const int i = tid + u * NT;
                        best[u] = i < count ? buf[i] : 0;
                        rank[u] = i < count ? rank_of<kBuf>(buf, count, best[u]) : kBuf;
                    }
                    sync();
#pragma unroll
                    for (int u = 0; u < kBuf / NT; ++u)
                        if (rank[u] < a.top) buf[rank[u]] = best[u];
                    if (tid == 0) count_s[slot][1] = min(count, a.top);
                    sync();
                    if (count >= a.top) bound = buf[a.top - 1];
                    count = min(count, a.top);
                }
            }
        }
        rank_out<NT, kBuf>(buf, count, a.top, tid, put);
    }
}

// The parts of a cut row, joined: a work-group to a row, a lane of every wave to a part.
template <typename T>
__global__ void __launch_bounds__(256)
token_logprobs_join_kernel(Args a) {
    constexpr int kKeys = kMaxSplit * kMaxTop, kPer = kKeys / 256;
    __shared__ key_t key_s[kKeys], buf[kKeys];
    __shared__ int count_s;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = lane_id();
    const int t = a.target ? a.target[row] : 0;
    Part st = {-INFINITY, 0.0f, 0.0f};
    if (lane < a.nsplit) st = a.part[row * a.nsplit + lane];
    // all keys of the row's parts, in registers and in LDS
    const key_t *keys = a.part_keys + row * a.nsplit * a.top;
    const int n = a.nsplit * a.top;
    key_t k[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) k[u] = tid + u * 256 < n ? keys[tid + u * 256] : 0;
    if (t < 0 || t >= a.V) {
        put_left_out(a, row, t, tid);
        return;
    }
    const float zt = tid == 0 ? Elem<T>::ld((const T *)a.logits + row * a.ld + t) : 0.0f;
    const float m = wave_max_nan(st.m);
    const float d = fmaxf((st.m - m) * a.c, -kFar), f = __builtin_amdgcn_exp2f(d);
    st = {m, wave_total(st.s * f), wave_total(fmaf(st.s, d, st.q) * f)};
    settle(st);
    const float ls = logf(st.s);
    if (a.top == 0 || !(m > -INFINITY && m < INFINITY)) {
        if (tid == 0) put_row(a, row, st, ls, zt);
        put_no_top(a, row, tid, m == -INFINITY ? -INFINITY : __uint_as_float(0x7fc00000u));
        return;
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u)
        if (tid + u * 256 < n) key_s[tid + u * 256] = k[u];
    if (tid == 0) count_s = 0;
    __syncthreads();
    // each part's keys come in descending order: what a.top of the 64 first ones over all parts reach bounds the row's
    const int p = lane % a.nsplit, at = lane / a.nsplit;
    const key_t first = at < a.top ? key_s[p * a.top + at] : 0;
    const float thr = reached_by(first ? key_logit(first) : -INFINITY, a.top);
#pragma unroll
    for (int u = 0; u < kPer; ++u)
        if (k[u] && key_logit(k[u]) >= thr) buf[atomicAdd(&count_s, 1)] = k[u];
    __syncthreads();
    rank_out<256, kKeys>(buf, count_s, a.top, tid, [&](int rank, key_t key) { put_top(a, row, rank, key, m, ls); });
    if (tid == 0) put_row(a, row, st, ls, zt);
}

constexpr int kGradLoads = 2;   // of 16 bytes, a thread's
struct BackArgs {
    int64_t row0, ld, ldd;
    int V, nseg, seg;
    float scale, c;
    const void *logits;
    const int32_t *target;
    const float *stats, *entropy, *dlogp, *dentropy;
    void *dlogits;
};

// A work-group to a piece of a row: NT threads with two loads each, all on their way at once, and gone after the stores.  Such
// short work-groups move 6.4 TB/s where pieces of four times the size moved 5.3 and a plain copy moves 5.4; stores are
// non-temporal, loads are not (8192 x 151936 bf16, a quarter left out, loads | stores: 712 us plain | plain, 670 plain | nt,
// 735 nt | nt, 702 nt | plain).  64 threads for rows of up to 2 KB: 16384 x 1000 bf16 13.0 us, with 256 18.1; rows of 4 KB
// 22.9 | 22.7.  With e = 2^x, x = c (z - m): dz = e (a + b x) + [v = t] s dlogp, where a = -(s / S) (dlogp + dH (H - log S)) and
// b = -(s / S) dH ln 2 are the row's.  dlogits may be logits: an element is read and written by one thread.
template <typename T, int NT, bool ENT>
__global__ void __launch_bounds__(NT)
token_logprobs_backward_kernel(BackArgs g) {
    typedef Row<T> R;
    constexpr int N = R::kVec;
    const int64_t row = g.row0 + blockIdx.x / g.nseg;
    const int lo = (int)(blockIdx.x % g.nseg) * g.seg, len = min(g.seg, g.V - lo);
    const T *z = (const T *)g.logits + row * g.ld + lo;
    T *dz = (T *)g.dlogits + row * g.ldd + lo;
    const int t = g.target ? g.target[row] : 0;
    const float m = g.stats[2 * row], S = g.stats[2 * row + 1];
    const bool live = t >= 0 && t < g.V && S != 0.0f;   // S = 0: every logit is -inf
    const float wt = g.dlogp ? g.dlogp[row] : 0.0f;
    float A = 0.0f, B = 0.0f;
    if (live) {
        const float r = -g.scale / S;
        A = wt;
        if constexpr (ENT) {
            const float dh = g.dentropy[row];
            A = fmaf(dh, g.entropy[row] - logf(S), wt);
            B = r * dh * kLn2;
        }
        A *= r;
    }
    const int at = live ? t - lo : -1 - N;   // the target's place here
    const float bonus = wt * g.scale;
    auto grad = [&](float v) {
        const float x = fmaxf((v - m) * g.c, -kFar), e = __builtin_amdgcn_exp2f(x);
        return e * (ENT ? fmaf(B, x, A) : A);
    };
    // vectors begin at 16-byte addresses of the gradient; a thread each for the elements before and behind them
    const int head = min(len, (int)((0 - (uintptr_t)dz) % 16 / sizeof(T))), nvec = (len - head) / N, rest = head + nvec * N;
    const int nloose = head + len - rest, atv = at - head;
    const T *zv = z + head;
    T *dv = dz + head;
    int j = threadIdx.x;
    if (live) {
        for (; j + (kGradLoads - 1) * NT < nvec; j += kGradLoads * NT) {
            typename R::V v[kGradLoads];
#pragma unroll
            for (int u = 0; u < kGradLoads; ++u) v[u] = R::load(zv + (int64_t)(j + u * NT) * N);
#pragma unroll
            for (int u = 0; u < kGradLoads; ++u) {
                float f[N];
                R::unpack(v[u], f);
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = grad(f[i]);
                const int rel = atv - (j + u * NT) * N;
                if (rel >= 0 && rel < N) {
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] = i == rel ? f[i] + bonus : f[i];
                }
                R::store_once(dv + (int64_t)(j + u * NT) * N, f);
            }
        }
    }
    for (; j < nvec; j += NT) {
        float f[N] = {};
        if (live) {
            R::unpack(R::load(zv + (int64_t)j * N), f);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = grad(f[i]) + (i == atv - j * N ? bonus : 0.0f);
        }
        R::store_once(dv + (int64_t)j * N, f);
    }
    if ((int)threadIdx.x < nloose) {
        const int i = (int)threadIdx.x < head ? threadIdx.x : rest + threadIdx.x - head;
        Elem<T>::st(dz + i, live ? grad(Elem<T>::ld(z + i)) + (i == at ? bonus : 0.0f) : 0.0f);
    }
}

// How a call cuts its rows: up to 128 of them, of 256 KB and more, into up to 512 work-groups in all, parts of 4096 elements at
// least (smaller ones do not shorten the chain of latencies that is left).  Others have 1024 threads and a compute unit each,
// which with 32 KB of loads on their way takes some 20 bytes a nanosecond, where a join and its launch cost 4 us and more.
// Cut | whole, bf16 with 20 alternatives: 96 rows of 66000 13.1 | 10.4 us, of 100000 13.6 | 12.4, of 151936 14.7 | 15.4, of
// 256000 16.8 | 21.9; 200 rows 14.8 | 10.9, 16.4 | 12.6, 19.5 | 15.2, 25.3 | 22.2.  512 | 1024 work-groups: 64 rows of 151936
// 13.5 | 14.0.
struct Plan {
    int nsplit, seg;
};
Plan plan(int64_t n, int64_t V, int elem_bytes) {
    constexpr int64_t kPart = 4096, kGroups = 512;
    if (n > 128 || V * elem_bytes < 262144) return {1, (int)V};
    const int64_t k = std::min(std::min<int64_t>(kGroups / n, kMaxSplit), (V + kPart - 1) / kPart);
    const int64_t seg = ((V + k - 1) / k + 7) / 8 * 8;
    return {(int)((V + seg - 1) / seg), (int)seg};
}
size_t part_bytes(int64_t n, const Plan &p) { return align_up((size_t)n * p.nsplit * sizeof(Part), 256); }

}  // namespace

size_t token_logprobs_ws_bytes(int64_t n, int64_t V, int top, int elem_bytes) {
    const Plan p = plan(n, V, elem_bytes);
    if (p.nsplit == 1) return 0;
    return part_bytes(n, p) + align_up((size_t)n * p.nsplit * top * sizeof(key_t), 256);
}

hipError_t launch_token_logprobs(int64_t n, int64_t V, int dtype, const void *logits, int64_t ld, float scale, const int32_t *target,
                                 float *logp, float *entropy, float *stats, int top, float *top_logp, int32_t *top_id, int32_t *status,
                                 void *ws, hipStream_t s) {
    const Plan p = plan(n, V, dtype == R3_BF16 ? 2 : 4);
    Args a = {};
    a.n = n; a.ld = ld; a.V = (int)V; a.top = top; a.nsplit = p.nsplit; a.seg = p.seg;
    a.scale = scale; a.c = (float)((double)scale * 1.4426950408889634); a.span = kSpan / a.c;
    a.logits = logits; a.target = target;
    a.logp = logp; a.entropy = entropy; a.stats = stats; a.top_logp = top_logp; a.top_id = top_id; a.status = status;
    if (p.nsplit > 1) {
        a.part = (Part *)ws;
        a.part_keys = (key_t *)((char *)ws + part_bytes(n, p));
    }
    ProfScope ps(PROF_LOGPROBS, s);
    auto go = [&](auto type, auto nt) {
        typedef decltype(type) T;
        constexpr int NT = decltype(nt)::value;
        auto k = top > 0 ? (entropy ? token_logprobs_kernel<T, NT, true, true> : token_logprobs_kernel<T, NT, false, true>)
                         : (entropy ? token_logprobs_kernel<T, NT, true, false> : token_logprobs_kernel<T, NT, false, false>);
        for (a.row0 = 0; a.row0 < n; a.row0 += kRowsAtOnce) {
            const int64_t rows = std::min<int64_t>(n - a.row0, kRowsAtOnce);
            k<<<(unsigned)(NT == kWave ? (rows + 3) / 4 : rows * p.nsplit), NT < 256 ? 256 : NT, 0, s>>>(a);
        }
        if (p.nsplit > 1) token_logprobs_join_kernel<T><<<(unsigned)n, 256, 0, s>>>(a);
    };
    auto by_size = [&](auto type) {
        const int64_t bytes = V * (int64_t)sizeof(type);
        const bool few = n <= 256 && p.nsplit == 1;   // a row has a compute unit to itself
        if (V <= 4096) go(type, std::integral_constant<int, 64>{});
        else if (bytes <= (few ? 16384 : top > 0 ? 131072 : 65536)) go(type, std::integral_constant<int, 256>{});
        else if (bytes <= 65536 || !few) go(type, std::integral_constant<int, 512>{});
        else go(type, std::integral_constant<int, 1024>{});
    };
    if (dtype == R3_BF16) by_size(bf16_t{});
    else by_size(float{});
    return hipGetLastError();
}

hipError_t launch_token_logprobs_backward(int64_t n, int64_t V, int dtype, const void *logits, int64_t ld, float scale,
                                          const int32_t *target, const float *stats, const float *entropy, const float *dlogp,
                                          const float *dentropy, void *dlogits, int64_t ldd, hipStream_t s) {
    BackArgs g = {};
    g.ld = ld; g.ldd = ldd; g.V = (int)V;
    g.scale = scale; g.c = (float)((double)scale * 1.4426950408889634);
    g.logits = logits; g.target = target; g.stats = stats; g.entropy = entropy; g.dlogp = dlogp; g.dentropy = dentropy; g.dlogits = dlogits;
    ProfScope ps(PROF_LOGPROBS_BWD, s);
    auto go = [&](auto type, auto nt) {
        typedef decltype(type) T;
        constexpr int NT = decltype(nt)::value;
        g.seg = kGradLoads * NT * Row<T>::kVec;
        g.nseg = (int)((V + g.seg - 1) / g.seg);
        auto k = dentropy ? token_logprobs_backward_kernel<T, NT, true> : token_logprobs_backward_kernel<T, NT, false>;
        const int64_t most = std::max<int64_t>(1, kRowsAtOnce / g.nseg);
        for (g.row0 = 0; g.row0 < n; g.row0 += most) k<<<(unsigned)(std::min(n - g.row0, most) * g.nseg), NT, 0, s>>>(g);
    };
    auto by_size = [&](auto type) {
        if (V * (int64_t)sizeof(type) <= 2048) go(type, std::integral_constant<int, 64>{});
        else go(type, std::integral_constant<int, 256>{});
    };
    if (dtype == R3_BF16) by_size(bf16_t{});
    else by_size(float{});
    return hipGetLastError();
}

}  // namespace r3
