// The losses of a training step with their gradients: the clipped policy loss over packed sequences, and the load-balance loss of the
// recorded routing with the router's z-loss.
//
// Sums over sequences.  Tokens are cut into pieces of equal length; the part of sequence q in piece p is segment p + q: on the way through
// the tokens every border raises one of the two, so no two segments that hold tokens share a number, and there are at most pieces +
// sequences of them, whatever the lengths are.  Each segment's sums are made by one work-group and added up over a sequence's segments in
// their order, so results are the same bits every time.  seq_start is only trusted to be ascending: positions are held within [0, n].
#include <algorithm>
#include <cmath>

#include "r3_kernels.h"
#include "r3_vec.h"

namespace r3 {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t lesser(int64_t a, int64_t b) { return a < b ? a : b; }
__device__ __forceinline__ int64_t larger(int64_t a, int64_t b) { return a > b ? a : b; }

// Sequences of a call: nseq of them, or one with everything.
struct Seqs {
    const int32_t *start;
    int nseq;
    int64_t n;
    __device__ __forceinline__ int64_t first(int q) const {
        if (!start) return q > 0 ? n : 0;
        const int64_t v = start[q];
        return v < 0 ? 0 : v > n ? n : v;
    }
    // The sequences that hold positions t0 and t1, the same in all lanes: the last that starts at or before each; -1 before the first,
    // nseq behind the last.  64 starts are looked at together, so that a search of 4096 takes two trips to memory.
    __device__ __forceinline__ void of(int64_t t0, int64_t t1, int &q0, int &q1) const {
        q0 = q1 = 0;
        if (!start) return;
        const int lane = threadIdx.x & (kWave - 1);
        int lo0 = -1, hi0 = nseq + 1, lo1 = -1, hi1 = nseq + 1;   // start[lo] <= t < start[hi]
        while (hi0 - lo0 > 1 || hi1 - lo1 > 1) {
            const int d0 = (hi0 - lo0 - 1 + kWave - 1) / kWave, d1 = (hi1 - lo1 - 1 + kWave - 1) / kWave;
            const int64_t i0 = lo0 + (int64_t)d0 * (lane + 1), i1 = lo1 + (int64_t)d1 * (lane + 1);
            const bool in0 = i0 < hi0, in1 = i1 < hi1;
            const int32_t s0 = start[in0 ? i0 : 0], s1 = start[in1 ? i1 : 0];
            // (starts ascend: the lanes that hold are the first ones)
            const int n0 = __popcll(__ballot(in0 && s0 <= t0)), n1 = __popcll(__ballot(in1 && s1 <= t1));
            if (hi0 - lo0 > 1) {
                const int64_t up = lo0 + (int64_t)d0 * (n0 + 1);
                lo0 += d0 * n0;
                hi0 = up < hi0 ? (int)up : hi0;
            }
            if (hi1 - lo1 > 1) {
                const int64_t up = lo1 + (int64_t)d1 * (n1 + 1);
                lo1 += d1 * n1;
                hi1 = up < hi1 ? (int)up : hi1;
            }
        }
        q0 = lo0;
        q1 = lo1;
    }
};

// Sums over a work-group, in every thread; `room`: as many values as it has waves.
template <int NT, typename T> __device__ __forceinline__ T block_sum(T v, T *room) {
    v = wave_sum(v);
    __syncthreads();
    if (lane_id() == 0) room[threadIdx.x / kWave] = v;
    __syncthreads();
    T s = room[0];
#pragma unroll
    for (int i = 1; i < NT / kWave; ++i) s += room[i];
    return s;
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Policy loss.  Of a live token with d = logp - old (a sequence's mean of it where ratios are a sequence's), r = e^d:
//   A > 0: used = min(r, 1 + high); A < 0: used = min(max(r, 1 - low), dual);  l = -w A used + kl k3(ref - logp) - ent H
//   w = min(e^(old - infer), cap);  k3(q) = e^q - 1 - q
//   dl/dlogp = -w A r where used = r, else 0, + kl (1 - e^q).  A sequence's ratio: the sum of the first part over its tokens, divided by
//   their number, to each of them.
// Which side of a border a token lies on is decided on d in 64 bits, where the difference of two floats is exact.  Two passes (the first
// reads only `target` unless ratios are a sequence's): tokens' weights need the numbers of live tokens.  Nothing but loads: the card is
// never busy, launches and their latencies are the time up to some 100 K tokens (us: one work-group's 1531 tokens 10, 64 K in 64 sequences
// 5 + 8.5 + 3, 1 M in 2048 with all terms 12.5 + 4 + 17 + 4, where the 17 move 38 MB at 2.2 TB/s; the 12.5 read 4 MB, a piece's sequences one after
// another, each two trips for its borders and targets and a sum with two barriers).  The sums' last launch as the end of the
// tokens' (the last work-group to come adds all up): no faster at 64 K, 27 us instead of 21 at 1 M, as many counters' turns.
// ---------------------------------------------------------------------------------------------------------------------------------

struct SegSum {      // of a segment
    double d, pos, neg;   // sums of d, and of w A over A > 0 and A < 0 (sequence ratios)
    int64_t live;
};
struct SeqOut {      // of a sequence
    double live;
    float up, down;  // what the ratio counts as for A > 0 and A < 0 (sequence ratios)
    float grad;      // and the policy's part of a token's gradient
    int cut;         // bit 0: cut for A > 0, bit 1: for A < 0
};
enum { kPolicySums = 5 };   // policy, kl, entropy, cut, weights
struct PolicyTotals { double live, seqs; };   // of some of the sequences

struct Policy {
    Seqs q;
    int piece, npieces;
    int norm;
    bool seq_ratio, adv_seq, kl_counts, ent_counts;
    const float *logp, *old, *infer, *ref, *entropy, *adv;
    const int32_t *target;
    float *dlogp, *dentropy, *stats;
    int32_t *status;
    double log_up, log_down, log_dual;   // borders of d
    float up, down, dual, cap, kl, ent, scale;
    SegSum *seg;
    SeqOut *seq;
    PolicyTotals *tot;
    int ntot;
    double *part;    // [npieces][kPolicySums]
};

// A token's values.  All of them are on their way before the first is used, kAhead tokens of a thread at a time: nothing else keeps the
// card busy here.
constexpr int kAhead = 4;
struct Token {
    float x, old, infer, A, ref, H;
    bool live;
};
template <bool ALL> __device__ __forceinline__ Token token(const Policy &a, int q, int64_t t, int64_t end) {
    Token k = {};
    k.live = t < end;
    const int64_t i = k.live ? t : end - 1;
    if (a.target) k.live &= a.target[i] >= 0;
    if (!ALL && !a.seq_ratio) return k;
    k.x = a.logp[i];
    k.old = a.old ? a.old[i] : k.x;
    k.A = a.adv[a.adv_seq ? q : i];
    if (a.infer) k.infer = a.infer[i];
    if (ALL && a.ref) k.ref = a.ref[i];
    if (ALL && a.entropy) k.H = a.entropy[i];
    return k;
}
__device__ __forceinline__ float weight(const Policy &a, const Token &k) {
    return a.infer ? __builtin_elementwise_minimum(expf(k.old - k.infer), a.cap) : 1.0f;   // (a NaN stays one)
}

// (without logp_old an infinite logp has d = 0, too; a NaN stays one)
__device__ __forceinline__ double log_ratio(const Policy &a, const Token &k) {
    return a.old || !isinf(k.x) ? (double)k.x - (double)k.old : 0.0;
}

// f(q, begin, end, all) for every segment of [lo, hi) of sequences q0 .. q1: all NT threads to each of a few, a wave to each of many
template <int NT, class F> __device__ __forceinline__ void for_segments(const Seqs &s, int64_t lo, int64_t hi, int q0, int q1, F f) {
    const bool few = q1 - q0 < 4;
    for (int q = few ? q0 : q0 + (int)threadIdx.x / kWave; q <= q1; q += few ? 1 : NT / kWave)
        f(q, larger(lo, s.first(q)), lesser(hi, s.first(q + 1)), few);
}
// sequences of a piece, one at least (that may hold none of its tokens)
__device__ __forceinline__ void of_piece(const Seqs &s, int64_t lo, int64_t hi, int &q0, int &q1) {
    s.of(lo, hi - 1, q0, q1);
    q0 = q0 < 0 ? 0 : q0 < s.nseq ? q0 : s.nseq - 1;
    q1 = q1 < q0 ? q0 : q1 < s.nseq ? q1 : s.nseq - 1;
}

// this thread's part of the sums over tokens b + first, + step, ... < e of sequence q
__device__ __forceinline__ SegSum segment_part(const Policy &a, int q, int64_t b, int64_t e, int first, int step) {
    SegSum s = {0.0, 0.0, 0.0, 0};
    if (!a.target && !a.seq_ratio) {      // (nothing to read)
        if (first == 0 && b < e) s.live = e - b;
        return s;
    }
    for (int64_t t = b + first; t < e; t += kAhead * step) {
        Token k[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) k[u] = token<false>(a, q, t + u * step, e);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (!k[u].live) continue;
            ++s.live;
            if (!a.seq_ratio) continue;
            s.d += log_ratio(a, k[u]);
            const float wA = k[u].A == 0.0f ? 0.0f : weight(a, k[u]) * k[u].A;   // (without an advantage the weight does not matter)
            if (k[u].A < 0.0f) s.neg += wA;
            else s.pos += wA;      // (or a NaN)
        }
    }
    return s;
}
__device__ __forceinline__ void over_wave_sums(const Policy &a, SegSum &x) {
    x.live = wave_sum((int)x.live);     // (at most 2^31 tokens)
    if (!a.seq_ratio) return;
    x.d = wave_sum(x.d);
    x.pos = wave_sum(x.pos);
    x.neg = wave_sum(x.neg);
}
__device__ __forceinline__ void add_sums(SegSum &x, const SegSum &y) {
    x.d += y.d;
    x.pos += y.pos;
    x.neg += y.neg;
    x.live += y.live;
}
// over a work-group, in thread 0; `room`: as many as it has waves
template <int NT> __device__ __forceinline__ void over_block_sums(const Policy &a, SegSum &x, SegSum *room) {
    over_wave_sums(a, x);
    __syncthreads();
    if (lane_id() == 0) room[threadIdx.x / kWave] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < NT / kWave; ++w) add_sums(x, room[w]);
}
// what follows from a sequence's sums
__device__ __forceinline__ SeqOut sequence_result(const Policy &a, const SegSum &s) {
    SeqOut o = {(double)s.live, 0.0f, 0.0f, 0.0f, 0};
    if (a.seq_ratio && s.live > 0) {
        const double d = s.d / (double)s.live;
        const float r = expf((float)d);
        const bool up = d > a.log_up, down = d < a.log_down, much = d > a.log_dual;
        o.up = up ? a.up : r;
        o.down = much ? a.dual : down ? a.down : r;
        o.cut = (up ? 1 : 0) | (down || much ? 2 : 0);
        // (nothing that the clip leaves free: no gradient, however large r is)
        const double free = (up ? 0.0 : s.pos) + (down || much ? 0.0 : s.neg);
        o.grad = free == 0.0 ? 0.0f : (float)(-(double)r * free / (double)s.live);
    }
    return o;
}
// a token's weight in the loss; all: live tokens, and sequences that hold them
__device__ __forceinline__ float token_weight(const Policy &a, double live_in_seq, const PolicyTotals &all) {
    if (live_in_seq == 0.0) return 0.0f;
    return (float)(a.norm == R3_MEAN_TOKENS ? a.scale / all.live : a.norm == R3_MEAN_SEQUENCES ? a.scale / (all.seqs * live_in_seq) : a.scale);
}

__global__ void __launch_bounds__(kThreads) policy_segments_kernel(Policy a) {
    __shared__ SegSum room[kThreads / kWave];
    const int p = blockIdx.x;
    const int64_t lo = (int64_t)p * a.piece, hi = lesser(lo + a.piece, a.q.n);
    int q0, q1;
    of_piece(a.q, lo, hi, q0, q1);
    for_segments<kThreads>(a.q, lo, hi, q0, q1, [&](int q, int64_t b, int64_t e, bool all) {
        SegSum s = segment_part(a, q, b, e, all ? (int)threadIdx.x : lane_id(), all ? kThreads : kWave);
        if (all) over_block_sums<kThreads>(a, s, room);
        else over_wave_sums(a, s);
        if ((all ? (int)threadIdx.x : lane_id()) == 0 && b < e) a.seg[(int64_t)p + q] = s;
    });
}

// Sequences' sums from their segments', to a wave each or (many) a thread each and a wave to those of many segments.
template <bool MANY> __global__ void __launch_bounds__(kThreads) policy_sequences_kernel(Policy a) {
    __shared__ PolicyTotals room[kThreads / kWave];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    // where sequence q's segments are, and how many
    auto segments = [&](int q, int64_t &at, int &n) {
        const int64_t b = a.q.first(q), e = a.q.first(q + 1);
        at = b < e ? b / a.piece + q : 0;
        n = b < e ? (int)((e - 1) / a.piece) + q - at + 1 : 0;
    };
    PolicyTotals t = {0.0, 0.0};
    auto done = [&](int q, const SegSum &s) {
        a.seq[q] = sequence_result(a, s);
        t.live += (double)s.live;
        t.seqs += s.live > 0;
    };
    int64_t at = 0;
    int n = 0;
    SegSum s = {0.0, 0.0, 0.0, 0};
    if constexpr (!MANY) {
        const int q = blockIdx.x * (kThreads / kWave) + wave;
        if (q < a.q.nseq) {
            segments(q, at, n);
            for (int i = lane; i < n; i += kWave) add_sums(s, a.seg[at + i]);
            over_wave_sums(a, s);
            if (lane == 0) done(q, s);
        }
    } else {
        constexpr int kFew = 4;
        const int q = blockIdx.x * kThreads + threadIdx.x;
        if (q < a.q.nseq) segments(q, at, n);
        if (n <= kFew)
            for (int i = 0; i < n; ++i) add_sums(s, a.seg[at + i]);
        for (uint64_t many = __ballot(n > kFew); many; many &= many - 1) {
            const int who = __builtin_ctzll(many), m = __shfl(n, who);
            const int64_t f = __shfl(at, who);
            SegSum w = {0.0, 0.0, 0.0, 0};
            for (int i = lane; i < m; i += kWave) add_sums(w, a.seg[f + i]);
            over_wave_sums(a, w);
            if (lane == who) s = w;
        }
        if (q < a.q.nseq) done(q, s);
    }
    t.live = wave_sum(t.live);
    t.seqs = wave_sum(t.seqs);
    if (lane == 0) room[wave] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / kWave; ++w) {
            t.live += room[w].live;
            t.seqs += room[w].seqs;
        }
        a.tot[blockIdx.x] = t;
    }
}

// Both at once, a work-group to a sequence, where even one that holds all tokens is gone through soon enough.
__global__ void __launch_bounds__(1024) policy_whole_kernel(Policy a) {
    __shared__ SegSum room[1024 / kWave];
    const int q = blockIdx.x;
    SegSum s = segment_part(a, q, a.q.first(q), a.q.first(q + 1), threadIdx.x, 1024);
    over_block_sums<1024>(a, s, room);
    if (threadIdx.x == 0) {
        a.seq[q] = sequence_result(a, s);
        a.tot[q] = {(double)s.live, s.live > 0 ? 1.0 : 0.0};
    }
}

// All live tokens and sequences, in every thread.
template <int NT> __device__ PolicyTotals policy_totals(const Policy &a, PolicyTotals *room) {
    PolicyTotals t = {0.0, 0.0};
    for (int i = threadIdx.x; i < a.ntot; i += NT) {
        t.live += a.tot[i].live;
        t.seqs += a.tot[i].seqs;
    }
    t.live = wave_sum(t.live);
    t.seqs = wave_sum(t.seqs);
    if (lane_id() == 0) room[threadIdx.x / kWave] = t;
    __syncthreads();
    t = room[0];
    for (int w = 1; w < NT / kWave; ++w) {
        t.live += room[w].live;
        t.seqs += room[w].seqs;
    }
    return t;
}

// A thread's part of the loss.
struct PolicyPart {
    double sum[kPolicySums] = {};
    bool bad = false;
    // live or not: token t, of a sequence with result s, weighing nu
    __device__ __forceinline__ void take(const Policy &a, int64_t t, const Token &k, const SeqOut &s, float nu) {
        float g = 0.0f;
        if (k.live) {
            const float A = k.A, w = weight(a, k), wA = w * A;
            float used;
            bool cut;
            if (a.seq_ratio) {
                used = A > 0.0f ? s.up : s.down;
                cut = A > 0.0f ? s.cut & 1 : A < 0.0f ? s.cut & 2 : false;
                g = s.grad;
            } else {
                const double d = log_ratio(a, k);
                const float r = expf((float)d);
                const bool up = d > a.log_up, down = d < a.log_down, over = d > a.log_dual;
                used = A > 0.0f ? (up ? a.up : r) : over ? a.dual : down ? a.down : r;
                cut = A > 0.0f ? up : A < 0.0f ? down || over : false;
                g = cut || A == 0.0f ? 0.0f : -wA * r;
            }
            float l = A == 0.0f ? 0.0f : -wA * used;
            sum[0] += (double)nu * l;
            // e^x - 1 - x: its leading terms where they cancel (the next is 2e-10 of them)
            auto third = [](float x, float ex) {
                const double y = x;
                return fabsf(x) < 0.125f ? y * y * (1.0 / 2 + y * (1.0 / 6 + y * (1.0 / 24 + y * (1.0 / 120 + y * (1.0 / 720 + y * (1.0 / 5040))))))
                                         : (double)ex - y;
            };
            // (a term with coefficient 0 is a statistic alone; a branch inside one that counts costs 1 M tokens 1.4 us)
            if (a.kl_counts) {
                const float x = k.ref - k.x, ex = expm1f(x);
                const double k3 = third(x, ex);
                sum[1] += (double)nu * k3;
                g = fmaf(-a.kl, ex, g);
                l += a.kl * (float)k3;
            } else if (a.ref) {
                const float x = k.ref - k.x;
                sum[1] += (double)nu * third(x, expm1f(x));
            }
            if (a.ent_counts) {
                sum[2] += (double)nu * k.H;
                l -= a.ent * k.H;
            } else if (a.entropy) sum[2] += (double)nu * k.H;
            sum[3] += cut;
            sum[4] += w;
            g *= nu;
            bad |= !isfinite(l) || !isfinite(g);
        }
        if (a.dlogp) a.dlogp[t] = g;
        if (a.dentropy) a.dentropy[t] = k.live ? -a.ent * nu : 0.0f;
    }
};
// Sequences of a piece that fit into LDS: a piece of as many or fewer is gone through once, whatever its borders are.
constexpr int kLocal = 128;
struct Local {
    SeqOut seq[kLocal];
    float nu[kLocal];
    int border[kLocal + 1];      // where they begin, from the piece's first token
};
// tokens lo .. hi - 1 of n sequences from q0 on, those outside [begin, end) of none
template <int NT>
__device__ __forceinline__ void policy_pass(const Policy &a, const Local &local, int q0, int n, int64_t lo, int64_t hi, int64_t begin, int64_t end, PolicyPart &part) {
    for (int64_t t = lo + threadIdx.x; t < hi; t += kAhead * NT) {
        Token k[kAhead];
        int at[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t i = lesser(t + u * NT, hi - 1);
            int x = 0, y = n;      // border[x] <= i - lo < border[y]
            while (y - x > 1) {
                const int m = (x + y) >> 1;
                if (local.border[m] <= (int)(i - lo)) x = m;
                else y = m;
            }
            at[u] = x;
            k[u] = {};
            if (i >= begin && i < end) k[u] = token<true>(a, q0 + x, i, hi);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (t + u * NT < hi) part.take(a, t + u * NT, k[u], local.seq[at[u]], local.nu[at[u]]);
    }
}
// the parts over a work-group, in the first kPolicySums threads
template <int NT> __device__ __forceinline__ double policy_sum(PolicyPart &part, double (*room)[kPolicySums]) {
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) part.sum[i] = wave_sum(part.sum[i]);
    if (lane_id() == 0)
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) room[threadIdx.x / kWave][i] = part.sum[i];
    __syncthreads();
    double v = 0.0;
    if (threadIdx.x < kPolicySums)
        for (int i = 0; i < NT / kWave; ++i) v += room[i][threadIdx.x];
    return v;
}
__device__ __forceinline__ void policy_report(const Policy &a, const PolicyPart &part) {
    if (a.status && __any(part.bad) && lane_id() == 0) atomicOr(a.status, R3_DATA_NONFINITE);
}

__global__ void __launch_bounds__(kThreads) policy_tokens_kernel(Policy a) {
    __shared__ double room[kThreads / kWave][kPolicySums];
    __shared__ PolicyTotals troom[kThreads / kWave];
    __shared__ Local local;
    const int64_t lo = (int64_t)blockIdx.x * a.piece, hi = lesser(lo + a.piece, a.q.n);
    int q0, q1;
    of_piece(a.q, lo, hi, q0, q1);
    const int n = q1 - q0 + 1;
    const int64_t begin = a.q.first(0), end = a.q.first(a.q.nseq);
    const PolicyTotals all = policy_totals<kThreads>(a, troom);
    PolicyPart part;
    if (n <= kLocal) {
        for (int i = threadIdx.x; i <= n; i += kThreads) {
            local.border[i] = (int)(larger(lo, lesser(hi, a.q.first(q0 + i))) - lo);
            if (i < n) {
                local.seq[i] = a.seq[q0 + i];
                local.nu[i] = token_weight(a, local.seq[i].live, all);
            }
        }
        __syncthreads();
        policy_pass<kThreads>(a, local, q0, n, lo, hi, begin, end, part);
    } else {
        for (int64_t t = lo + threadIdx.x; t < hi; t += kThreads)
            if (t < begin || t >= end) part.take(a, t, Token{}, SeqOut{}, 0.0f);
        for_segments<kThreads>(a.q, lo, hi, q0, q1, [&](int q, int64_t b, int64_t e, bool) {
            if (b >= e) return;
            const SeqOut s = a.seq[q];
            const float nu = token_weight(a, s.live, all);
            for (int64_t t = b + lane_id(); t < e; t += kWave) part.take(a, t, token<true>(a, q, t, e), s, nu);
        });
    }
    const double v = policy_sum<kThreads>(part, room);
    if (threadIdx.x < kPolicySums) a.part[(int64_t)blockIdx.x * kPolicySums + threadIdx.x] = v;
    policy_report(a, part);
}

// the loss and its parts, from the sums
__device__ __forceinline__ void policy_stats(const Policy &a, const double (&v)[kPolicySums], const PolicyTotals &all) {
    const double some = all.live > 0.0 ? all.live : 1.0, unit = a.scale != 0.0f ? 1.0 / a.scale : 0.0;
    a.stats[0] = (float)(v[0] + (a.kl_counts ? (double)a.kl * v[1] : 0.0) - (a.ent_counts ? (double)a.ent * v[2] : 0.0));
    a.stats[1] = (float)v[0];
    a.stats[2] = (float)(v[1] * unit);
    a.stats[3] = (float)(v[2] * unit);
    a.stats[4] = (float)(v[3] / some);
    a.stats[5] = (float)(v[4] / some);
    a.stats[6] = (float)all.live;
    a.stats[7] = (float)all.seqs;
}
__global__ void __launch_bounds__(kThreads) policy_finish_kernel(Policy a) {
    __shared__ double room[kThreads / kWave][kPolicySums], total[kPolicySums];
    __shared__ PolicyTotals troom[kThreads / kWave];
    PolicyPart part;
    for (int p = threadIdx.x; p < a.npieces; p += kThreads)
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) part.sum[i] += a.part[(int64_t)p * kPolicySums + i];
    const double s = policy_sum<kThreads>(part, room);
    if (threadIdx.x < kPolicySums) total[threadIdx.x] = s;
    const PolicyTotals all = policy_totals<kThreads>(a, troom);
    __syncthreads();
    if (threadIdx.x > 0) return;
    double v[kPolicySums];
    for (int i = 0; i < kPolicySums; ++i) v[i] = total[i];
    policy_stats(a, v, all);
}

// One work-group does it all, with the sequences in LDS.
constexpr int kSmallThreads = 512;
constexpr int64_t kPolicySmall = 4096;
__global__ void __launch_bounds__(kSmallThreads) policy_small_kernel(Policy a) {
    __shared__ double room[kSmallThreads / kWave][kPolicySums], total[kPolicySums];
    __shared__ SegSum sroom[kSmallThreads / kWave];
    __shared__ Local local;
    const int n = a.q.nseq;
    const int64_t begin = a.q.first(0), end = a.q.first(n);
    for (int i = threadIdx.x; i <= n; i += kSmallThreads) local.border[i] = (int)a.q.first(i);
    __syncthreads();
    if (n <= 2) {
        for (int q = 0; q < n; ++q) {
            SegSum s = segment_part(a, q, local.border[q], local.border[q + 1], threadIdx.x, kSmallThreads);
            over_block_sums<kSmallThreads>(a, s, sroom);
            if (threadIdx.x == 0) local.seq[q] = sequence_result(a, s);
        }
    } else {
        for (int q = threadIdx.x / kWave; q < n; q += kSmallThreads / kWave) {
            SegSum s = segment_part(a, q, local.border[q], local.border[q + 1], lane_id(), kWave);
            over_wave_sums(a, s);
            if (lane_id() == 0) local.seq[q] = sequence_result(a, s);
        }
    }
    __syncthreads();
    PolicyTotals all = {0.0, 0.0};
    for (int q = 0; q < n; ++q) {
        all.live += local.seq[q].live;
        all.seqs += local.seq[q].live > 0.0;
    }
    for (int q = threadIdx.x; q < n; q += kSmallThreads) local.nu[q] = token_weight(a, local.seq[q].live, all);
    __syncthreads();
    PolicyPart part;
    policy_pass<kSmallThreads>(a, local, 0, n, 0, a.q.n, begin, end, part);
    const double s = policy_sum<kSmallThreads>(part, room);
    if (threadIdx.x < kPolicySums) total[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double v[kPolicySums];
        for (int i = 0; i < kPolicySums; ++i) v[i] = total[i];
        policy_stats(a, v, all);
    }
    policy_report(a, part);
}

struct PolicyPlan {
    int piece, npieces, ntot;
    bool small, whole, many;
    size_t seg, seq, tot, part, total;
};
PolicyPlan policy_plan(int64_t n, int nseq) {
    PolicyPlan p;
    p.small = n <= kPolicySmall && nseq <= kLocal;
    // a work-group to a sequence: 128 tokens to a thread if one has them all
    p.whole = n <= 131072 && nseq >= 8 && nseq <= 4096;
    p.many = nseq > 4096;
    p.ntot = p.whole ? nseq : p.many ? (nseq + kThreads - 1) / kThreads : (nseq + kThreads / kWave - 1) / (kThreads / kWave);
    // at least two tokens to a thread, and at most 1024 work-groups until a piece has 8192
    const int64_t piece = align_up((size_t)((n + 1023) / 1024), kThreads);
    p.piece = (int)std::min<int64_t>(std::max<int64_t>(piece, 2 * kThreads), 8192);
    p.npieces = (int)((n + p.piece - 1) / p.piece);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    p.seg = take(p.whole ? 0 : ((size_t)p.npieces + nseq) * sizeof(SegSum));
    p.seq = take((size_t)nseq * sizeof(SeqOut));
    p.tot = take((size_t)p.ntot * sizeof(PolicyTotals));
    p.part = take((size_t)p.npieces * kPolicySums * sizeof(double));
    p.total = o;
    return p;
}

}  // namespace

size_t policy_loss_ws_bytes(int64_t n, int nseq) { return policy_plan(n, nseq < 1 ? 1 : nseq).total; }

hipError_t launch_policy_loss(const r3_policy_desc &D, const float *logp, const float *old, const float *infer, const float *ref,
                              const float *entropy, const float *adv, const int32_t *target, const int32_t *seq_start, float *dlogp,
                              float *dentropy, float *stats, int32_t *status, void *ws, hipStream_t s) {
    ProfScope ps(PROF_POLICY_LOSS, s);
    const int nseq = seq_start ? D.nseq : 1;
    const PolicyPlan p = policy_plan(D.n, nseq);
    char *base = (char *)ws;
    Policy a = {};
    a.q = {seq_start, nseq, D.n};
    a.piece = p.piece; a.npieces = p.npieces;
    a.norm = D.norm; a.seq_ratio = D.ratio == R3_RATIO_SEQUENCE; a.adv_seq = (D.flags & R3_FLAG_SEQ_ADVANTAGE) != 0;
    a.logp = logp; a.old = old; a.infer = infer; a.ref = ref; a.entropy = entropy; a.adv = adv; a.target = target;
    a.dlogp = dlogp; a.dentropy = dentropy; a.stats = stats; a.status = status;
    a.up = 1.0f + D.clip_high; a.down = 1.0f - D.clip_low; a.dual = D.dual_clip;
    a.log_up = std::log1p((double)D.clip_high);
    a.log_down = D.clip_low < 1.0f ? std::log1p(-(double)D.clip_low) : -INFINITY;
    a.log_dual = D.dual_clip > 0.0f ? std::log((double)D.dual_clip) : INFINITY;
    a.kl_counts = D.kl_coef != 0.0f; a.ent_counts = D.entropy_coef != 0.0f;
    a.cap = D.weight_cap; a.kl = D.kl_coef; a.ent = D.entropy_coef; a.scale = D.scale;
    a.seg = (SegSum *)(base + p.seg); a.seq = (SeqOut *)(base + p.seq); a.tot = (PolicyTotals *)(base + p.tot); a.part = (double *)(base + p.part);
    a.ntot = p.ntot;
    if (p.small) {
        policy_small_kernel<<<1, kSmallThreads, 0, s>>>(a);
        return hipGetLastError();
    }
    if (p.whole) policy_whole_kernel<<<nseq, 1024, 0, s>>>(a);
    else {
        if (p.npieces) policy_segments_kernel<<<p.npieces, kThreads, 0, s>>>(a);
        (p.many ? policy_sequences_kernel<true> : policy_sequences_kernel<false>)<<<p.ntot, kThreads, 0, s>>>(a);
    }
    if (p.npieces) policy_tokens_kernel<<<p.npieces, kThreads, 0, s>>>(a);
    policy_finish_kernel<<<1, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

namespace {

// ---------------------------------------------------------------------------------------------------------------------------------
// Load-balance loss.  Of group g (a sequence, or the batch) with N tokens and c_e slots recorded for expert e: f_e = E c_e / (K N),
// p_t = softmax of token t's logits; loss = alpha mean_g mean_t sum_e f_e p_te + zeta mean_t lse_t^2.
//   ds_te = alpha / (groups N) p_te (f_e - sum_i f_i p_ti) + 2 zeta / tokens lse_t p_te
// The counts come from the record alone, a byte or two to a slot, so they are made first and the logits are read once: a token's
// probabilities give its part of the loss and its gradient at once.  HBM-bound where it counts: 65536 x 128 counts 4, join 3, tokens 16 us
// (67 MB at 4.2 TB/s), finish 4; 131072 x 128 in 64 sequences 8 + 4 + 31 + 4; 3001 x 384 in 7 4 + 13 + 3, latencies.
// ---------------------------------------------------------------------------------------------------------------------------------

struct Balance {
    Seqs q;
    int T, E, K;
    int piece0, npieces0;      // of the counts
    int piece, npieces;        // of the logits
    bool once;                 // dlogits is more than the caches may hold for who reads it (131072 x 128 marked | not 28.6 | 32.3 us, 65536 16.3 | 16.6)
    const void *idx;
    int64_t stride;            // of a token's record
    const float *logits;
    int64_t ld, ldd;
    float alpha, zeta;
    int32_t *counts;           // [groups, E]
    float *probs, *stats, *dlogits;   // (probs, dlogits: or none)
    int32_t *status;
    int32_t *hist;             // [segments of pieces0, E]
    float *psum;               // [segments, E]
    double *lsum;              // [pieces][2]: sums of f p, each over its group's tokens, and of lse^2
    double *tot;               // groups that hold tokens, tokens
};

// The record's counts of tokens b .. e - 1, to `to`.  Ids that lie one behind the other are read 16 bytes at a time.  COPIES: lanes that meet
// in an expert have up to eight histograms, their counts of it in different banks, in kMaxE counts (a work-group's 240000 slots of 128 experts
// 54 | 38 us a call, 32000 of 8 20 | 14; 4000 or 8000 of a piece's 0.5 longer, so pieces have one).
template <int NT, bool COPIES, typename IdxT> __device__ __forceinline__ void balance_count(const Balance &a, int64_t b, int64_t e, int *hist, int32_t *to, bool &bad) {
    const int copies = !COPIES ? 1 : a.E < kMaxE / 8 ? 8 : a.E < kMaxE / 4 ? 4 : a.E < kMaxE / 2 ? 2 : 1, apart = copies > 1 ? a.E + 1 : a.E;
    for (int i = threadIdx.x; i < copies * apart; i += NT) hist[i] = 0;
    __syncthreads();
    int *mine = hist + (threadIdx.x & (copies - 1)) * apart;
    const IdxT *idx = (const IdxT *)a.idx + b * a.stride;
    const int n = b < e ? (int)(e - b) * a.K : 0;
    auto one = [&](int id) {
        if (id < a.E) atomicAdd(&mine[id], 1);
        else bad = true;
    };
    if (a.stride == a.K) {
        constexpr int kVec = 16 / (int)sizeof(IdxT);
        const int head = (int)lesser(n, ((16 - (int)((uintptr_t)idx & 15)) & 15) / (int)sizeof(IdxT)), vecs = (n - head) / kVec;
        for (int i = threadIdx.x; i < vecs; i += NT) {
            const uint4 v = ((const uint4 *)(idx + head))[i];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int u = 0; u < kVec; ++u) one((int)((w[u * (int)sizeof(IdxT) / 4] >> (8 * (int)sizeof(IdxT) * u % 32)) & ((1u << 8 * sizeof(IdxT)) - 1)));
        }
        const int rest = n - vecs * kVec;     // in front and behind
        for (int i = threadIdx.x; i < rest; i += NT) one(idx[i < head ? i : i + vecs * kVec]);
    } else {
        for (int i = threadIdx.x; i < n; i += NT) {
            const int t = i / a.K;
            one(idx[(int64_t)t * a.stride + (i - t * a.K)]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.E; i += NT) {
        int n = hist[i];
        for (int k = 1; k < copies; ++k) n += hist[k * apart + i];
        to[i] = n;
    }
}
__device__ __forceinline__ void balance_report(const Balance &a, bool bad) {
    if (a.status && bad) atomicOr(a.status, R3_DATA_IDX_RANGE);
}
// in each segment of piece p
template <int NT, typename IdxT> __device__ void balance_counts(const Balance &a, int p, int *hist) {
    const int64_t lo = (int64_t)p * a.piece0, hi = lesser(lo + a.piece0, a.T);
    bool bad = false;
    if (lo < hi) {
        int q0, q1;
        of_piece(a.q, lo, hi, q0, q1);
        for (int q = q0; q <= q1; ++q) {
            const int64_t b = larger(lo, a.q.first(q)), e = lesser(hi, a.q.first(q + 1));
            if (b >= e) continue;
            balance_count<NT, false, IdxT>(a, b, e, hist, a.hist + (int64_t)(p + q) * a.E, bad);
            __syncthreads();
        }
    }
    balance_report(a, bad);
}
// groups and tokens, by one work-group
template <int NT> __device__ void balance_totals(const Balance &a, double *room) {
    double some = 0.0;
    for (int q = threadIdx.x; q < a.q.nseq; q += NT) some += a.q.first(q) < a.q.first(q + 1);
    some = block_sum<NT>(some, room);
    if (threadIdx.x == 0) {
        a.tot[0] = some;
        a.tot[1] = (double)(a.q.first(a.q.nseq) - a.q.first(0));
    }
}

template <typename IdxT> __global__ void __launch_bounds__(1024) balance_counts_kernel(Balance a) {
    __shared__ int hist[kMaxE];
    __shared__ double room[1024 / kWave];
    balance_counts<1024, IdxT>(a, blockIdx.x, hist);
    if (blockIdx.x == 0) balance_totals<1024>(a, room);
}

// A work-group to a group, and nothing to join, where even one that holds all tokens is gone through soon enough.
template <typename IdxT> __global__ void __launch_bounds__(1024) balance_whole_kernel(Balance a) {
    __shared__ int hist[kMaxE];
    __shared__ double room[1024 / kWave];
    const int q = blockIdx.x;
    bool bad = false;
    balance_count<1024, true, IdxT>(a, a.q.first(q), a.q.first(q + 1), hist, a.counts + (int64_t)q * a.E, bad);
    balance_report(a, bad);
    if (q == 0) balance_totals<1024>(a, room);
}

// A group's counts of 16 experts, 16 threads to each, segments in turn and then the 16 sums in their order
constexpr int kColumns = 16;
template <int NT> __device__ void balance_join(const Balance &a, int64_t item, int (*sums)[kColumns]) {
    constexpr int kRows = NT / kColumns;
    const int per = (a.E + kColumns - 1) / kColumns, q = (int)(item / per), l = threadIdx.x % kColumns, w = threadIdx.x / kColumns;
    const int c = (int)(item - (int64_t)q * per) * kColumns + l;
    const int64_t b = a.q.first(q), e = a.q.first(q + 1);
    int n = 0;
    if (b < e && c < a.E) {
        const int p0 = (int)(b / a.piece0), p1 = (int)((e - 1) / a.piece0);
#pragma unroll 4
        for (int p = p0 + w; p <= p1; p += kRows) n += a.hist[(int64_t)(p + q) * a.E + c];
    }
    __syncthreads();
    sums[w][l] = n;
    __syncthreads();
    if (w > 0 || c >= a.E) return;
    n = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) n += sums[i][l];
    a.counts[(int64_t)q * a.E + c] = n;
}
__device__ __forceinline__ int64_t balance_items(const Balance &a) { return (int64_t)a.q.nseq * ((a.E + kColumns - 1) / kColumns); }
__global__ void __launch_bounds__(kThreads) balance_join_kernel(Balance a) {
    __shared__ int sums[kThreads / kColumns][kColumns];
    for (int64_t i = blockIdx.x, n = balance_items(a); i < n; i += gridDim.x) balance_join<kThreads>(a, i, sums);
}

// A value over L neighbouring lanes, in all of them: within 16 by moves in the vector pipe (pairs, pairs of pairs, mirrored halves of 8 and
// 16)
template <int L, class F> __device__ __forceinline__ float over_lanes(float v, F f) {
    if constexpr (L >= 2) v = f(v, lane_move<0xb1, 0xf>(v, v));
    if constexpr (L >= 4) v = f(v, lane_move<0x4e, 0xf>(v, v));
    if constexpr (L >= 8) v = f(v, lane_move<0x141, 0xf>(v, v));
    if constexpr (L >= 16) v = f(v, lane_move<0x140, 0xf>(v, v));
    if constexpr (L >= 32) v = f(v, __shfl_xor(v, 16, kWave));
    if constexpr (L >= 64) v = f(v, __shfl_xor(v, 32, kWave));
    return v;
}

// A token to L lanes, V vectors of four logits to a lane: lane l of them has columns 4 (l + L v) .. + 3.  The next token's logits are on
// their way while one is worked on.
template <int NT, int L, int V> __device__ void balance_tokens(const Balance &a, int p) {
    constexpr int kTok = NT / L;       // tokens at a time
    __shared__ float sums[kTok][L * 4];
    __shared__ double room[NT / kWave];
    const int64_t lo = (int64_t)p * a.piece, hi = lesser(lo + a.piece, a.T);
    const int l = threadIdx.x % L, w = threadIdx.x / L;
    int qa, qb;
    a.q.of(lo, hi - 1, qa, qb);
    double tf = 0.0, tz = 0.0;       // this piece's part of the loss
    bool bad = false;
    auto columns = [&](int v) { const int c = 4 * (l + L * v); return c + 4 <= a.E ? 4 : a.E - c; };   // (none: 0 or less)
    auto load = [&](int64_t t, float (&x)[V][4]) {
        const float *z = a.logits + t * a.ld;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = columns(v), c = 4 * (l + L * v);
            if (n == 4) Row<float>::unpack(Row<float>::load(z + c), x[v]);
            else {
#pragma unroll
                for (int u = 0; u < 4; ++u) x[v][u] = u < n ? z[c + u] : -INFINITY;
            }
        }
    };
    for (int q = qa; q <= qb; ++q) {
        const bool none = q < 0 || q >= a.q.nseq;    // tokens of no sequence
        const int64_t b = q < 0 ? lo : larger(lo, a.q.first(q)), e = q < 0 ? lesser(hi, a.q.first(0)) : q >= a.q.nseq ? hi : lesser(hi, a.q.first(q + 1));
        if (b >= e) continue;
        if (none) {
            if (a.dlogits)
                for (int64_t t = b + w; t < e; t += kTok)
                    for (int c = l; c < a.E; c += L) a.dlogits[t * a.ldd + c] = 0.0f;
            continue;
        }
        const double len = (double)(a.q.first(q + 1) - a.q.first(q));
        const float share = (float)((double)a.E / (a.K * len)), ga = (float)(a.alpha / (a.tot[0] * len)), gz = (float)(2.0 * a.zeta / a.tot[1]);
        float x[V][4];
        if (b + w < e) load(b + w, x);
        float f[V][4], acc[V][4];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                f[v][u] = u < columns(v) ? (float)a.counts[(int64_t)q * a.E + 4 * (l + L * v) + u] * share : 0.0f;
                acc[v][u] = 0.0f;
            }
        double sf = 0.0;
        for (int64_t t = b + w; t < e; t += kTok) {
            float next[V][4];
            if (t + kTok < e) load(t + kTok, next);
            float m = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int u = 0; u < 4; ++u) m = __builtin_elementwise_maximum(m, x[v][u]);
            m = over_lanes<L>(m, [](float i, float j) { return __builtin_elementwise_maximum(i, j); });
            const bool empty = m == -INFINITY;    // nothing but masked experts
            float S = 0.0f, dot = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    x[v][u] = empty ? 0.0f : __builtin_amdgcn_exp2f((x[v][u] - m) * 1.44269504088896f);
                    S += x[v][u];
                    dot = fmaf(f[v][u], x[v][u], dot);
                }
            S = over_lanes<L>(S, [](float i, float j) { return i + j; });
            dot = over_lanes<L>(dot, [](float i, float j) { return i + j; });
            // (1 <= S <= E; the hardware's reciprocal and logarithm are off by one unit in the last place)
            const float inv = empty ? 0.0f : __builtin_amdgcn_rcpf(S), mean = dot * inv;
            const float lse = empty ? 0.0f : fmaf(__builtin_amdgcn_logf(S), 0.693147180559945f, m), zg = gz * lse;
            bad |= !isfinite(mean + lse);
            if (l == 0) {
                sf += mean;
                tz += (double)lse * lse;
            }
            float *g = a.dlogits + t * a.ldd;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int n = columns(v), c = 4 * (l + L * v);
                float d[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float pr = x[v][u] * inv;
                    acc[v][u] += pr;
                    d[u] = pr * fmaf(ga, f[v][u] - mean, zg);
                }
                if (a.dlogits) {
                    if (n == 4) {
                        if (a.once) Row<float>::store_once(g + c, d);
                        else Row<float>::store(g + c, d);
                    } else
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (u < n) g[c + u] = d[u];
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int u = 0; u < 4; ++u) x[v][u] = next[v][u];
        }
        tf += sf / len;
        if (a.probs) {
            const int64_t seg = (int64_t)p + q;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                __syncthreads();
#pragma unroll
                for (int u = 0; u < 4; ++u) sums[w][4 * l + u] = acc[v][u];
                __syncthreads();
                const int c = threadIdx.x, at = 4 * L * v + c;
                if (c < 4 * L && at < a.E) {
                    float s = 0.0f;
#pragma unroll 8
                    for (int i = 0; i < kTok; ++i) s += sums[i][c];
                    a.psum[seg * a.E + at] = s;
                }
            }
        }
    }
    tf = block_sum<NT>(tf, room);
    tz = block_sum<NT>(tz, room);
    if (threadIdx.x == 0) {
        a.lsum[2 * (int64_t)p] = tf;
        a.lsum[2 * (int64_t)p + 1] = tz;
    }
    if (a.status && __any(bad) && lane_id() == 0) atomicOr(a.status, R3_DATA_NONFINITE);
}

template <int L, int V> __global__ void __launch_bounds__(kThreads) balance_tokens_kernel(Balance a) { balance_tokens<kThreads, L, V>(a, blockIdx.x); }

// The loss, by one work-group.
template <int NT> __device__ void balance_loss(const Balance &a, double *room) {
    double bal = 0.0, z = 0.0;
#pragma unroll 4
    for (int p = threadIdx.x; p < a.npieces; p += NT) {
        bal += a.lsum[2 * (int64_t)p];
        z += a.lsum[2 * (int64_t)p + 1];
    }
    bal = block_sum<NT>(bal, room);
    z = block_sum<NT>(z, room);
    if (threadIdx.x == 0) {
        const double some = a.tot[0] > 0.0 ? a.tot[0] : 1.0, n = a.tot[1] > 0.0 ? a.tot[1] : 1.0;
        a.stats[0] = (float)((double)a.alpha * bal / some + (double)a.zeta * z / n);
        a.stats[1] = (float)(bal / some);
        a.stats[2] = (float)(z / n);
    }
}

// Mean probabilities of 16 experts of a group, as balance_join
template <int NT> __device__ void balance_probs(const Balance &a, int64_t item, double (*sums)[kColumns]) {
    constexpr int kRows = NT / kColumns;
    const int per = (a.E + kColumns - 1) / kColumns, q = (int)(item / per), l = threadIdx.x % kColumns, w = threadIdx.x / kColumns;
    const int c = (int)(item - (int64_t)q * per) * kColumns + l;
    const int64_t b = a.q.first(q), e = a.q.first(q + 1);
    double s = 0.0;
    if (b < e && c < a.E) {
        const int p0 = (int)(b / a.piece), p1 = (int)((e - 1) / a.piece);
#pragma unroll 8
        for (int p = p0 + w; p <= p1; p += kRows) s += a.psum[(int64_t)(p + q) * a.E + c];
    }
    __syncthreads();
    sums[w][l] = s;
    __syncthreads();
    if (w > 0 || c >= a.E) return;
    s = 0.0;
#pragma unroll 8
    for (int i = 0; i < kRows; ++i) s += sums[i][l];
    a.probs[(int64_t)q * a.E + c] = b < e ? (float)(s / (double)(e - b)) : 0.0f;
}

// the first work-group: the loss
template <int NT> __global__ void __launch_bounds__(NT) balance_finish_kernel(Balance a) {
    __shared__ double room[NT / kWave], sums[NT / kColumns][kColumns];
    if (blockIdx.x == 0) balance_loss<NT>(a, room);
    else
        for (int64_t i = blockIdx.x - 1, n = balance_items(a); i < n; i += gridDim.x - 1) balance_probs<NT>(a, i, sums);
}

// one work-group does it all, a step behind the other
constexpr int kSmallE = 256;
template <typename IdxT, int L> __global__ void __launch_bounds__(kThreads) balance_small_kernel(Balance a) {
    __shared__ int hist[kSmallE];
    __shared__ double room[kThreads / kWave], dsum[kThreads / kColumns][kColumns];
    __shared__ int isum[kThreads / kColumns][kColumns];
    balance_counts<kThreads, IdxT>(a, 0, hist);
    balance_totals<kThreads>(a, room);
    __syncthreads();
    for (int64_t i = 0, n = balance_items(a); i < n; ++i) balance_join<kThreads>(a, i, isum);
    __syncthreads();
    balance_tokens<kThreads, L, 1>(a, 0);
    __syncthreads();
    balance_loss<kThreads>(a, room);
    if (a.probs)
        for (int64_t i = 0, n = balance_items(a); i < n; ++i) balance_probs<kThreads>(a, i, dsum);
}

// One work-group up to 16 K logits of few groups.
bool balance_small(int64_t T, int E, int nseq) { return E <= kSmallE && T * E <= 16384 && T <= 512 && (int64_t)nseq * E <= 1024; }

// A work-group to a group saves the join of pieces: up to 32768 slots of one, 65536 of two, and 262144 of 32 and more, which seldom are one's (us
// a call, pieces | whole: 4000 x 128, 8 slots 16.3 | 16.0, 1000 14.3 | 12.3; two groups of 8000 20.5 | 18.6, all in one 19.5 | 19.1; 64 of 32000
// 31 | 24, all in one 28 | 42; 300 of 32000 x 64, 6 slots 34 | 22).
bool balance_whole(int64_t T, int K, int nseq) {
    return nseq <= 4096 && T * K <= 32768 * (int64_t)(nseq >= 32 ? 8 : std::min(nseq, 2));
}

struct BalancePlan {
    int piece0, npieces0, piece, npieces;
    size_t hist, psum, lsum, tot, counts, total;
};
BalancePlan balance_plan(int64_t T, int E, int nseq) {
    BalancePlan p;
    // counts: at most 128 work-groups of 1024 threads, as one group's join adds up a part of each.  (Many groups have few parts each whatever the
    // limit is: half of the card idles then, 7.8 us for the 1 MB of 131072 x 8 in 64.)
    p.piece0 = (int)std::max<int64_t>((T + 127) / 128, 128);
    // logits: 16 KB and more to a work-group, at most 1024 of them (65536 x 128: 16.6 us; 2048 of them, whose beginnings and ends count,
    // 20.3)
    p.piece = (int)std::max<int64_t>((T + 1023) / 1024, std::max<int64_t>(4, 4096 / E));
    if (balance_small(T, E, nseq)) p.piece0 = p.piece = (int)T;
    p.npieces0 = (int)((T + p.piece0 - 1) / p.piece0);
    p.npieces = (int)((T + p.piece - 1) / p.piece);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    p.hist = take(((size_t)p.npieces0 + nseq) * E * sizeof(int32_t));
    p.psum = take(((size_t)p.npieces + nseq) * E * sizeof(float));
    p.lsum = take((size_t)p.npieces * 2 * sizeof(double));
    p.tot = take(2 * sizeof(double));
    p.counts = take((size_t)nseq * E * sizeof(int32_t));
    p.total = o;
    return p;
}

}  // namespace

size_t balance_loss_ws_bytes(int64_t T, int E, int nseq) { return balance_plan(T, E, nseq < 1 ? 1 : nseq).total; }

hipError_t launch_balance_loss(int T, int E, int K, const float *logits, int64_t ld, const void *idx, int idx_dtype, int64_t stride,
                               const int32_t *seq_start, int nseq, float alpha, float zeta, int32_t *counts, float *probs, float *stats,
                               float *dlogits, int64_t ldd, int32_t *status, void *ws, hipStream_t s) {
    ProfScope ps(PROF_BALANCE_LOSS, s);
    if (!seq_start) nseq = 1;
    const BalancePlan p = balance_plan(T, E, nseq);
    char *base = (char *)ws;
    Balance a = {};
    a.q = {seq_start, nseq, T};
    a.T = T; a.E = E; a.K = K;
    a.once = (int64_t)T * E * (int64_t)sizeof(float) > 48 << 20;
    a.piece0 = p.piece0; a.npieces0 = p.npieces0; a.piece = p.piece; a.npieces = p.npieces;
    a.idx = idx; a.stride = stride; a.logits = logits; a.ld = ld; a.ldd = ldd; a.alpha = alpha; a.zeta = zeta;
    a.counts = counts ? counts : (int32_t *)(base + p.counts); a.probs = probs; a.stats = stats; a.dlogits = dlogits; a.status = status;
    a.hist = (int32_t *)(base + p.hist); a.psum = (float *)(base + p.psum); a.lsum = (double *)(base + p.lsum); a.tot = (double *)(base + p.tot);
    const int vecs = (E + 3) / 4;
    const bool u8 = idx_dtype == R3_IDX_U8;
    auto lanes = [&](auto go) {     // of a token
        if (vecs <= 2) go(std::integral_constant<int, 2>{});
        else if (vecs <= 4) go(std::integral_constant<int, 4>{});
        else if (vecs <= 8) go(std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, 16>{});
    };
    if (balance_small(T, E, nseq)) {
        auto go = [&](auto l) {
            constexpr int L = decltype(l)::value;
            if (u8) balance_small_kernel<uint8_t, L><<<1, kThreads, 0, s>>>(a);
            else balance_small_kernel<uint16_t, L><<<1, kThreads, 0, s>>>(a);
        };
        if (vecs <= 16) lanes(go);
        else if (vecs <= 32) go(std::integral_constant<int, 32>{});
        else go(std::integral_constant<int, 64>{});
        return hipGetLastError();
    }
    const int64_t items = (int64_t)nseq * ((E + kColumns - 1) / kColumns), most = 1 << 20;
    if (balance_whole(T, K, nseq)) {
        if (u8) balance_whole_kernel<uint8_t><<<nseq, 1024, 0, s>>>(a);
        else balance_whole_kernel<uint16_t><<<nseq, 1024, 0, s>>>(a);
    } else {
        if (u8) balance_counts_kernel<uint8_t><<<p.npieces0, 1024, 0, s>>>(a);
        else balance_counts_kernel<uint16_t><<<p.npieces0, 1024, 0, s>>>(a);
        balance_join_kernel<<<(unsigned)std::min(items, most), kThreads, 0, s>>>(a);
    }
    auto go = [&](auto l, auto v) { balance_tokens_kernel<decltype(l)::value, decltype(v)::value><<<p.npieces, kThreads, 0, s>>>(a); };
    typedef std::integral_constant<int, 64> wave;
    if (vecs <= 16) lanes([&](auto l) { go(l, std::integral_constant<int, 1>{}); });
    else if (vecs <= 32) go(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    else if (vecs <= 64) go(std::integral_constant<int, 32>{}, std::integral_constant<int, 2>{});
    else if (vecs <= 128) go(std::integral_constant<int, 32>{}, std::integral_constant<int, 4>{});
    else if (vecs <= 256) go(wave{}, std::integral_constant<int, 4>{});
    else if (vecs <= 512) go(wave{}, std::integral_constant<int, 8>{});
    else go(wave{}, std::integral_constant<int, 16>{});
    // (of one group's many pieces each column is a long sum)
    const unsigned grid = (unsigned)(1 + (probs ? std::min(items, most) : 0));
    if (p.npieces / nseq > 256) balance_finish_kernel<1024><<<grid, 1024, 0, s>>>(a);
    else balance_finish_kernel<kThreads><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace r3
