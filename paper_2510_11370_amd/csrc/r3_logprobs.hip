// Log-probabilities of given tokens, entropy and the most probable alternatives of a row of logits, and the gradient:
//   x_v = s (z_v - m), m = max z;  S = sum e^x;  log p_v = x_v - log S;  H = log S - (sum e^x x) / S
//   dz_v = s ([v = t] dlogp - p_v (dlogp + dH (log p_v + H)))
// Both read the logits once (and the gradient writes once): HBM-bound.
#include <algorithm>

#include "r3_kernels.h"
#include "r3_vec.h"

namespace r3 {
namespace {

constexpr int kMaxTop = R3_MAX_TOP;
constexpr int kMaxSplit = 64;       // parts of a row: one lane each when they are joined
constexpr float kFar = 1e4f;        // 2^-kFar is 0: exponents are kept above -kFar, so that 0 x (-inf) never arises
constexpr int64_t kRowsAtOnce = 1 << 22;   // work-groups of a launch: a grid has less than 2^32 threads
constexpr float kLn2 = 0.693147180559945309f;

// The larger of two numbers; NaN if one is NaN (v_maximum3_f32), so that a row's maximum says whether it holds one.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_max_nan(float v) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o, kWave));
    return v;
}

// Running statistics over some of a row's elements: m their maximum, s = sum 2^x, q = sum 2^x x with
// x = c (z - m), c = s log2(e).  m = -inf, s = q = 0: nothing yet, or nothing but -inf.
struct Stat {
    float m, s, q;
};
// the same sums for another maximum, which is at least a.m (or NaN)
template <bool ENT> __device__ __forceinline__ void rebase(Stat &a, float m, float c) {
    const float d = fmaxf((a.m - m) * c, -kFar), f = __builtin_amdgcn_exp2f(d);   // (-inf less -inf: -kFar, f = 0)
    if constexpr (ENT) a.q = fmaf(a.s, d, a.q) * f;
    a.s *= f;
    a.m = m;
}

// N more elements.
template <int N, bool ENT> __device__ __forceinline__ void take(Stat &a, const float (&z)[N], float c) {
    float hi = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) hi = max_nan(hi, z[i]);
    rebase<ENT>(a, max_nan(a.m, hi), c);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = fmaxf((z[i] - a.m) * c, -kFar), e = __builtin_amdgcn_exp2f(x);
        a.s += e;
        if constexpr (ENT) a.q = fmaf(e, x, a.q);
    }
}

// A logit and its place in one whole number: larger logits first, then lower places.  0: none.
typedef unsigned long long key_t;
__device__ __forceinline__ key_t make_key(float z, int v) {
    const uint32_t b = __float_as_uint(z + 0.0f);   // -0 equals +0
    const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return ((key_t)o << 32) | (0xffffffffu - (uint32_t)v);
}
__device__ __forceinline__ float key_logit(key_t k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_place(key_t k) { return (int)(0xffffffffu - (uint32_t)k); }

struct Args {
    int64_t n, ld, row0;            // rows row0 .. n - 1
    int V, top, nsplit, seg;        // seg: elements of one part of a row
    float scale, c;
    const void *logits;
    const int32_t *target;
    float *logp, *entropy, *stats, *top_logp;
    int32_t *top_id, *status;
    Stat *part;                     // [n][nsplit], and
    key_t *part_keys;               // [n][nsplit][top], where rows are cut
};

// scale (z - m), of halves: z - m itself may be past the range where scale < 1
__device__ __forceinline__ float log_odds(float z, float m, float scale) {
    const float d = (0.5f * z - 0.5f * m) * scale;
    return d + d;
}

// What a row comes to, by the thread that has it.
__device__ __forceinline__ void put_row(const Args &a, int64_t row, const Stat &r, float zt) {
    const float ls = logf(r.s), nan = __uint_as_float(0x7fc00000u);
    const bool bad = !(r.m < INFINITY), none = r.m == -INFINITY;
    if (bad && a.status) atomicOr(a.status, R3_DATA_NONFINITE);
    if (a.logp) a.logp[row] = bad ? nan : none ? -INFINITY : log_odds(zt, r.m, a.scale) - ls;
    if (a.entropy) a.entropy[row] = bad ? nan : none ? 0.0f : ls - r.q * kLn2 / r.s;
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

// Of the candidates in buf[0..count) the `top` largest, each to its rank; keys are distinct (0 is none).
template <int NT, class F> __device__ __forceinline__ void rank_out(const key_t *buf, int count, int top, int tid, F put) {
    for (int i = tid; i < count; i += NT) {
        const key_t k = buf[i];
        int rank = 0;
        for (int q = 0; q < count; ++q) rank += buf[q] > k;
        if (rank < top) put(rank, k);
    }
    for (int i = count + tid; i < top; i += NT) put(i, (key_t)0);
}

// The k-th largest of the lanes' values: each lane counts those above its own, and the smallest value with less than k
// above it is the one.
__device__ __forceinline__ float kth_of_wave(float v, int k) {
    int above = 0;
#pragma unroll 8
    for (int i = 0; i < kWave; ++i) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), i)) > v;
    float t = above < k ? v : INFINITY;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) t = fminf(t, __shfl_xor(t, o, kWave));
    return t;
}

// NT threads to a row (or to one of a.nsplit parts of it); NT = 64: four rows to a work-group, nothing shared between its
// waves.
//
// Alternatives: a thread knows the maximum of its own elements anyway.  The 64 maxima over the threads of one lane number
// are 64 elements of the row, so the k-th largest of them has k elements at or above it: a bound from below for the k-th
// largest element, met by some 64 ln(64 / (64 - k)) elements of a row in random order (24 for k = 20).  Only the threads
// whose maximum reaches it are read again, by whole waves, from L2.  Rows that keep more candidates than fit (many equal
// values) are gone through once more in order with the k-th best so far as the bound.
template <typename T, int NT, bool ENT, bool TOP>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT)
token_logprobs_kernel(Args a) {
    typedef Row<T> R;
    constexpr int N = R::kVec, U = 4, W = NT / kWave, kRows = NT == kWave ? 4 : 1;
    constexpr int kBuf = 2 * NT;   // room for the k best and one more element from every thread
    static_assert(kBuf >= NT + kMaxTop, "");
    __shared__ float max_s[kRows][W][kWave], sum_s[kRows][2][W], thr_s[kRows];
    __shared__ int count_s[kRows][2];
    __shared__ int sel_s[TOP ? kRows : 1][TOP ? NT : 1];
    __shared__ key_t buf_s[TOP ? kRows : 1][TOP ? kBuf : 1];
    const int lane = lane_id(), slot = kRows > 1 ? (int)threadIdx.x / kWave : 0;
    const int tid = kRows > 1 ? lane : (int)threadIdx.x, w = tid / kWave;
    auto sync = [] {
        if constexpr (W > 1) __syncthreads();
        else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    const int64_t item = a.row0 * a.nsplit + (int64_t)blockIdx.x * kRows + slot;
    const int64_t row = item / a.nsplit;
    const int split = (int)(item - row * a.nsplit);
    if (row >= a.n) return;
    const int t = a.target ? a.target[row] : 0;
    if (t < 0 || t >= a.V) {
        if (split == 0) put_left_out(a, row, t, tid);
        return;
    }
    const T *z = (const T *)a.logits + row * a.ld;
    const int lo = split * a.seg, len = min(a.seg, a.V - lo), nvec = len / N;
    const T *zp = z + lo;
    float zt = 0.0f;
    if (tid == 0) {
        zt = Elem<T>::ld(z + t);
        count_s[slot][0] = count_s[slot][1] = 0;
    }
    Stat st = {-INFINITY, 0.0f, 0.0f};
    int j = tid;
    for (; j + (U - 1) * NT < nvec; j += U * NT) {
        typename R::V v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = R::load(zp + (int64_t)(j + u * NT) * N);
        float f[U * N];
#pragma unroll
        for (int u = 0; u < U; ++u) R::unpack(v[u], f + u * N);
        take<U * N, ENT>(st, f, a.c);
    }
    for (; j < nvec; j += NT) {
        float f[N];
        R::unpack(R::load(zp + (int64_t)j * N), f);
        take<N, ENT>(st, f, a.c);
    }
    if (tid < len - nvec * N) {
        const float f[1] = {Elem<T>::ld(zp + nvec * N + tid)};
        take<1, ENT>(st, f, a.c);
    }

    const float mine = st.m;
    float top64 = mine;   // the largest of the threads with this lane's number
    if constexpr (W > 1) {
        max_s[slot][w][lane] = mine;
        sync();
#pragma unroll
        for (int i = 0; i < W; ++i) top64 = max_nan(top64, max_s[slot][i][lane]);
    }
    const float m = wave_max_nan(top64);
    rebase<ENT>(st, m, a.c);
    st.s = wave_sum(st.s);
    if constexpr (ENT) st.q = wave_sum(st.q);
    if constexpr (W > 1) {
        if (lane == 0) {
            sum_s[slot][0][w] = st.s;
            sum_s[slot][1][w] = st.q;
        }
    }
    const bool search = TOP && m > -INFINITY && m < INFINITY;   // (the same in every thread)
    if (search && w == 0) {
        const float b = kth_of_wave(top64, a.top);
        if (lane == 0) thr_s[slot] = b;
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
    if (tid == 0) {
        if (a.nsplit == 1) put_row(a, row, st, zt);
        else a.part[item] = st;
    }
    if constexpr (TOP) {
        const float ls = logf(st.s);
        auto put = [&](int rank, key_t k) {
            if (a.nsplit == 1) put_top(a, row, rank, k, m, ls);
            else a.part_keys[item * a.top + rank] = k;
        };
        if (!search) {
            if (a.nsplit == 1) put_no_top(a, row, tid, m == -INFINITY ? -INFINITY : __uint_as_float(0x7fc00000u));
            else if (tid < a.top) a.part_keys[item * a.top + tid] = 0;
            return;
        }
        const float thr = thr_s[slot];
        int *sel = sel_s[slot];
        key_t *buf = buf_s[slot];
        if (mine >= thr && mine > -INFINITY) sel[atomicAdd(&count_s[slot][0], 1)] = tid;
        sync();
        const int nsel = count_s[slot][0];
        auto offer = [&](float x, int place) {
            if (x >= thr && x > -INFINITY) {
                const int at = atomicAdd(&count_s[slot][1], 1);
                if (at < kBuf) buf[at] = make_key(x, lo + place);
            }
        };
        for (int i = w; i < nsel; i += W) {
            const int who = sel[i];
            for (int q = who + lane * NT; q < nvec; q += kWave * NT) {
                float f[N];
                R::unpack(R::load(zp + (int64_t)q * N), f);
#pragma unroll
                for (int u = 0; u < N; ++u) offer(f[u], q * N + u);
            }
            if (lane == 0 && who < len - nvec * N) offer(Elem<T>::ld(zp + nvec * N + who), nvec * N + who);
        }
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
                        rank[u] = i < count ? 0 : kBuf;
                        for (int q = 0; q < count; ++q) rank[u] += buf[q] > best[u];
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
        rank_out<NT>(buf, count, a.top, tid, put);
    }
}

// The parts of a cut row, joined: a work-group to a row, a lane of every wave to a part.
template <typename T>
__global__ void __launch_bounds__(256)
token_logprobs_join_kernel(Args a) {
    __shared__ key_t buf[kMaxSplit * kMaxTop], head_s[kWave];
    __shared__ int count_s;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = lane_id();
    const int t = a.target ? a.target[row] : 0;
    if (t < 0 || t >= a.V) return;   // written by the row's first part
    Stat st = {-INFINITY, 0.0f, 0.0f};
    if (lane < a.nsplit) st = a.part[row * a.nsplit + lane];
    const float zt = tid == 0 ? Elem<T>::ld((const T *)a.logits + row * a.ld + t) : 0.0f;
    const float m = wave_max_nan(st.m);
    rebase<true>(st, m, a.c);
    st.s = wave_sum(st.s);
    st.q = wave_sum(st.q);
    if (tid == 0) put_row(a, row, st, zt);
    if (a.top == 0) return;
    if (!(m > -INFINITY && m < INFINITY)) {
        put_no_top(a, row, tid, m == -INFINITY ? -INFINITY : __uint_as_float(0x7fc00000u));
        return;
    }
    // each part's keys come in descending order: the k-th largest of the 64 first ones over all parts bounds the k-th
    // largest of all
    const key_t *keys = a.part_keys + row * a.nsplit * a.top;
    const int n = a.nsplit * a.top;
    if (tid == 0) count_s = 0;
    if (tid < kWave) {
        const int p = tid % a.nsplit, at = tid / a.nsplit;
        head_s[tid] = at < a.top ? keys[p * a.top + at] : 0;
    }
    __syncthreads();
    const key_t mine = head_s[lane];
    int above = 0;
    for (int i = 0; i < kWave; ++i) above += head_s[i] > mine;
    key_t thr = above < a.top ? mine : ~0ull;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
        const key_t other = __shfl_xor(thr, o, kWave);
        thr = other < thr ? other : thr;
    }
    for (int i = tid; i < n; i += 256) {
        const key_t k = keys[i];
        if (k && k >= thr) buf[atomicAdd(&count_s, 1)] = k;
    }
    __syncthreads();
    const float ls = logf(st.s);
    rank_out<256>(buf, count_s, a.top, tid, [&](int rank, key_t k) { put_top(a, row, rank, k, m, ls); });
}

struct BackArgs {
    int64_t row0, ld, ldd;
    int V, nseg, seg;
    float scale, c;
    const void *logits;
    const int32_t *target;
    const float *stats, *entropy, *dlogp, *dentropy;
    void *dlogits;
};

// A work-group to a piece of a row.  With e = 2^x, x = c (z - m): dz = e (a + b x) + [v = t] s dlogp, where
// a = -(s / S) (dlogp + dH (H - log S)) and b = -(s / S) dH ln 2 are the row's.  dlogits may be logits: an element is
// read and written by one thread.
template <typename T, bool ENT>
__global__ void __launch_bounds__(256)
token_logprobs_backward_kernel(BackArgs g) {
    typedef Row<T> R;
    constexpr int N = R::kVec;
    const int64_t row = g.row0 + blockIdx.x / g.nseg;
    const int lo = (int)(blockIdx.x % g.nseg) * g.seg, len = min(g.seg, g.V - lo), nvec = len / N;
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
    const int at = live ? t - lo : -1;   // the target's place here
    auto grad = [&](float v, int i) {
        const float x = fmaxf((v - m) * g.c, -kFar), e = __builtin_amdgcn_exp2f(x);
        const float d = e * (ENT ? fmaf(B, x, A) : A);
        return i == at ? fmaf(wt, g.scale, d) : d;
    };
    for (int j = threadIdx.x; j < nvec; j += 256) {
        float f[N];
        if (live) {
            R::unpack(R::load(z + (int64_t)j * N), f);
#pragma unroll
            for (int u = 0; u < N; ++u) f[u] = grad(f[u], j * N + u);
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) f[u] = 0.0f;
        }
        R::store(dz + (int64_t)j * N, f);
    }
    const int rest = nvec * N + threadIdx.x;
    if (rest < len) Elem<T>::st(dz + rest, live ? grad(Elem<T>::ld(z + rest), rest) : 0.0f);
}

// How a call cuts its rows.
struct Plan {
    int nsplit, seg;
};
Plan plan(int64_t n, int64_t V) {
    const int64_t least = 4096, want = n > 0 ? 1024 / n : 1;
    int64_t k = std::min<int64_t>(std::min<int64_t>(want, kMaxSplit), V / least);
    if (k <= 1) return {1, (int)V};
    const int64_t seg = ((V + k - 1) / k + 7) / 8 * 8;
    return {(int)((V + seg - 1) / seg), (int)seg};
}
size_t stat_bytes(int64_t n, const Plan &p) { return align_up((size_t)n * p.nsplit * sizeof(Stat), 256); }

}  // namespace

size_t token_logprobs_ws_bytes(int64_t n, int64_t V, int top) {
    const Plan p = plan(n, V);
    if (p.nsplit == 1) return 0;
    return stat_bytes(n, p) + align_up((size_t)n * p.nsplit * top * sizeof(key_t), 256);
}

hipError_t launch_token_logprobs(int64_t n, int64_t V, int dtype, const void *logits, int64_t ld, float scale, const int32_t *target,
                                 float *logp, float *entropy, float *stats, int top, float *top_logp, int32_t *top_id, int32_t *status,
                                 void *ws, hipStream_t s) {
    const Plan p = plan(n, V);
    Args a = {};
    a.n = n; a.ld = ld; a.V = (int)V; a.top = top; a.nsplit = p.nsplit; a.seg = p.seg;
    a.scale = scale; a.c = (float)((double)scale * 1.4426950408889634);
    a.logits = logits; a.target = target;
    a.logp = logp; a.entropy = entropy; a.stats = stats; a.top_logp = top_logp; a.top_id = top_id; a.status = status;
    if (p.nsplit > 1) {
        a.part = (Stat *)ws;
        a.part_keys = (key_t *)((char *)ws + stat_bytes(n, p));
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
        if (V <= 4096) go(type, std::integral_constant<int, 64>{});
        else if (V <= 32768) go(type, std::integral_constant<int, 256>{});
        else go(type, std::integral_constant<int, 512>{});
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
    g.seg = (int)std::min<int64_t>(V, 8192);
    g.nseg = (int)((V + g.seg - 1) / g.seg);
    g.scale = scale; g.c = (float)((double)scale * 1.4426950408889634);
    g.logits = logits; g.target = target; g.stats = stats; g.entropy = entropy; g.dlogp = dlogp; g.dentropy = dentropy; g.dlogits = dlogits;
    ProfScope ps(PROF_LOGPROBS_BWD, s);
    auto go = [&](auto type) {
        typedef decltype(type) T;
        auto k = dentropy ? token_logprobs_backward_kernel<T, true> : token_logprobs_backward_kernel<T, false>;
        const int64_t most = std::max<int64_t>(1, kRowsAtOnce / g.nseg);
        for (g.row0 = 0; g.row0 < n; g.row0 += most) k<<<(unsigned)(std::min(n - g.row0, most) * g.nseg), 256, 0, s>>>(g);
    };
    if (dtype == R3_BF16) go(bf16_t{});
    else go(float{});
    return hipGetLastError();
}

}  // namespace r3
