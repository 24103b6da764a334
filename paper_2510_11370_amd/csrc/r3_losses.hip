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
    // the sequence that holds position t: the last that starts at or before it; -1 before the first, nseq behind the last
    __device__ __forceinline__ int of(int64_t t) const {
        if (!start) return 0;
        int lo = -1, hi = nseq + 1;   // start[lo] <= t < start[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= t) lo = mid;
            else hi = mid;
        }
        return lo;
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
// reads only `target` unless ratios are a sequence's): tokens' weights need the numbers of live tokens.  Nothing but loads: the card
// is never busy, launches and their latencies are the time up to some 100 K tokens.
// ---------------------------------------------------------------------------------------------------------------------------------

struct SegSum {      // of a segment
    double d, pos, neg;   // sums of d, and of w A over A > 0 and A < 0 (sequence ratios)
    int64_t live;
};
struct SeqOut {      // of a sequence
    double live;
    float nu;        // a token's weight
    float up, down;  // what the ratio counts as for A > 0 and A < 0 (sequence ratios)
    float grad;      // and the policy's part of a token's gradient
    int cut;         // bit 0: cut for A > 0, bit 1: for A < 0
};
enum { kPolicySums = 5 };   // policy, kl, entropy, cut, weights
struct PolicyTotals { double live, seqs; };

struct Policy {
    Seqs q;
    int piece, npieces;
    int norm;
    bool seq_ratio, adv_seq;
    const float *logp, *old, *infer, *ref, *entropy, *adv;
    const int32_t *target;
    float *dlogp, *dentropy, *stats;
    int32_t *status;
    double log_up, log_down, log_dual;   // borders of d
    float up, down, dual, cap, kl, ent, scale;
    SegSum *seg;
    SeqOut *seq;
    PolicyTotals *tot;
    double *part;    // [npieces][kPolicySums]
};

__device__ __forceinline__ double log_ratio(const Policy &a, int64_t t) { return a.old ? (double)a.logp[t] - (double)a.old[t] : 0.0; }
__device__ __forceinline__ float weight(const Policy &a, int64_t t) {
    if (!a.infer) return 1.0f;
    return __builtin_elementwise_minimum(expf((a.old ? a.old[t] : a.logp[t]) - a.infer[t]), a.cap);   // (a NaN stays one)
}

__device__ __forceinline__ void seg_add(const Policy &a, int q, int64_t t, SegSum &s) {
    if (a.target && a.target[t] < 0) return;
    ++s.live;
    if (!a.seq_ratio) return;
    s.d += log_ratio(a, t);
    const float A = a.adv[a.adv_seq ? q : t], wA = weight(a, t) * A;
    if (A > 0.0f) s.pos += wA;
    else if (A < 0.0f) s.neg += wA;
    else s.pos += wA * 0.0f;   // (a NaN stays one)
}

template <int NT> __device__ void policy_segments(const Policy &a, int p) {
    __shared__ double room[NT / kWave];
    __shared__ int64_t iroom[NT / kWave];
    const int64_t lo = (int64_t)p * a.piece, hi = lesser(lo + a.piece, a.q.n);
    if (lo >= hi) return;
    int q0 = a.q.of(lo), q1 = a.q.of(hi - 1);
    q0 = q0 < 0 ? 0 : q0;
    q1 = q1 >= a.q.nseq ? a.q.nseq - 1 : q1;
    // few segments: all threads to each; many: a wave to each
    if (q1 - q0 < 4) {
        for (int q = q0; q <= q1; ++q) {
            const int64_t b = larger(lo, a.q.first(q)), e = lesser(hi, a.q.first(q + 1));
            SegSum s = {0.0, 0.0, 0.0, 0};
            for (int64_t t = b + threadIdx.x; t < e; t += NT) seg_add(a, q, t, s);
            s.live = block_sum<NT>(s.live, iroom);
            if (a.seq_ratio) {
                s.d = block_sum<NT>(s.d, room);
                s.pos = block_sum<NT>(s.pos, room);
                s.neg = block_sum<NT>(s.neg, room);
            }
            if (threadIdx.x == 0 && b < e) a.seg[p + q] = s;
        }
        return;
    }
    for (int q = q0 + (int)threadIdx.x / kWave; q <= q1; q += NT / kWave) {
        const int64_t b = larger(lo, a.q.first(q)), e = lesser(hi, a.q.first(q + 1));
        SegSum s = {0.0, 0.0, 0.0, 0};
        for (int64_t t = b + lane_id(); t < e; t += kWave) seg_add(a, q, t, s);
        s.live = wave_sum(s.live);
        if (a.seq_ratio) {
            s.d = wave_sum(s.d);
            s.pos = wave_sum(s.pos);
            s.neg = wave_sum(s.neg);
        }
        if (lane_id() == 0 && b < e) a.seg[p + q] = s;
    }
}

// One work-group: sequences' sums, what follows from them, and the numbers of live tokens and sequences.
template <int NT> __device__ void policy_sequences(const Policy &a) {
    __shared__ double room[NT / kWave];
    const int lane = lane_id();
    double live = 0.0, seqs = 0.0;
    for (int base = 0; base < a.q.nseq; base += NT) {
        const int q = base + threadIdx.x;
        int64_t b = 0, e = 0;
        if (q < a.q.nseq) {
            b = a.q.first(q);
            e = a.q.first(q + 1);
        }
        const int s0 = b < e ? (int)(b / a.piece) : 0, ns = b < e ? (int)((e - 1) / a.piece) - s0 + 1 : 0;
        SegSum s = {0.0, 0.0, 0.0, 0};
        constexpr int kFew = 8;
        auto add = [](SegSum &x, const SegSum &y) {
            x.d += y.d;
            x.pos += y.pos;
            x.neg += y.neg;
            x.live += y.live;
        };
        if (ns <= kFew)
            for (int i = 0; i < ns; ++i) add(s, a.seg[s0 + q + i]);
        // a long sequence's segments to a wave
        for (uint64_t many = __ballot(ns > kFew); many; many &= many - 1) {
            const int who = __builtin_ctzll(many), f = __shfl(s0 + q, who), n = __shfl(ns, who);
            SegSum w = {0.0, 0.0, 0.0, 0};
            for (int i = lane; i < n; i += kWave) add(w, a.seg[f + i]);
            w.d = wave_sum(w.d);
            w.pos = wave_sum(w.pos);
            w.neg = wave_sum(w.neg);
            w.live = wave_sum(w.live);
            if (lane == who) s = w;
        }
        if (q < a.q.nseq) {
            SeqOut o = {(double)s.live, 0.0f, 0.0f, 0.0f, 0.0f, 0};
            if (a.seq_ratio && s.live > 0) {
                const double d = s.d / (double)s.live;
                const float r = expf((float)d);
                const bool up = d > a.log_up, down = d < a.log_down, over = d > a.log_dual;
                o.up = up ? a.up : r;
                o.down = over ? a.dual : down ? a.down : r;
                o.cut = (up ? 1 : 0) | (down || over ? 2 : 0);
                o.grad = (float)(-(double)r * ((up ? 0.0 : s.pos) + (down || over ? 0.0 : s.neg)) / (double)s.live);
            }
            a.seq[q] = o;
            live += (double)s.live;
            seqs += s.live > 0;
        }
    }
    live = block_sum<NT>(live, room);
    seqs = block_sum<NT>(seqs, room);
    for (int q = threadIdx.x; q < a.q.nseq; q += NT) {
        const double n = a.seq[q].live;
        a.seq[q].nu = n == 0.0 ? 0.0f : (float)(a.norm == R3_MEAN_TOKENS ? a.scale / live : a.norm == R3_MEAN_SEQUENCES ? a.scale / (seqs * n) : a.scale);
    }
    if (threadIdx.x == 0) *a.tot = {live, seqs};
}

struct PolicyIn {
    float logp, old, infer, ref, entropy, adv;
    bool live;
};

template <int NT> __device__ void policy_tokens(const Policy &a, int p) {
    __shared__ double room[NT / kWave];
    const int64_t lo = (int64_t)p * a.piece, hi = lesser(lo + a.piece, a.q.n);
    const int64_t begin = a.q.first(0), end = a.q.first(a.q.nseq);
    double sum[kPolicySums] = {};
    bool bad = false;
    const int qa = lo < hi ? a.q.of(lo) : 0, qb = lo < hi ? a.q.of(hi - 1) : 0;
    for (int64_t t = lo + threadIdx.x; t < hi; t += NT) {
        const bool live = t >= begin && t < end && !(a.target && a.target[t] < 0);
        const int q = qa == qb ? qa : a.q.of(t);
        float g = 0.0f, gh = 0.0f;
        if (live && q >= 0 && q < a.q.nseq) {
            const SeqOut s = a.seq[q];
            const float A = a.adv[a.adv_seq ? q : t], w = weight(a, t), wA = w * A, x = a.logp[t];
            float used;
            bool cut;
            if (a.seq_ratio) {
                used = A > 0.0f ? s.up : s.down;
                cut = A > 0.0f ? s.cut & 1 : A < 0.0f ? s.cut & 2 : false;
                g = s.grad;
            } else {
                const double d = log_ratio(a, t);
                const float r = expf((float)d);
                const bool up = d > a.log_up, down = d < a.log_down, over = d > a.log_dual;
                used = A > 0.0f ? (up ? a.up : r) : over ? a.dual : down ? a.down : r;
                cut = A > 0.0f ? up : A < 0.0f ? down || over : false;
                g = cut ? 0.0f : -wA * r;
            }
            const float l = A == 0.0f ? 0.0f : -wA * used;
            if (A == 0.0f && !a.seq_ratio) g = 0.0f;
            float all = l;
            sum[0] += (double)s.nu * l;
            if (a.ref) {
                const float k = a.ref[t] - x, e = expm1f(k);
                // e^q - 1 - q: its leading terms where they cancel
                const double k3 = fabsf(k) < 0.125f ? (double)k * k * (0.5 + (double)k * (1.0 / 6 + (double)k * (1.0 / 24 + (double)k * (1.0 / 120 + (double)k * (1.0 / 720 + (double)k * (1.0 / 5040)))))) : (double)e - k;
                sum[1] += (double)s.nu * k3;
                g = fmaf(-a.kl, e, g);
                all += a.kl * (float)k3;
            }
            if (a.entropy) {
                const float H = a.entropy[t];
                sum[2] += (double)s.nu * H;
                all -= a.ent * H;
            }
            sum[3] += cut;
            sum[4] += w;
            g *= s.nu;
            gh = -a.ent * s.nu;
            bad |= !isfinite(all) || !isfinite(g);
        }
        if (a.dlogp) a.dlogp[t] = g;
        if (a.dentropy) a.dentropy[t] = gh;
    }
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) {
        const double v = block_sum<NT>(sum[i], room);
        if (threadIdx.x == 0) a.part[(int64_t)p * kPolicySums + i] = v;
    }
    if (a.status && __any(bad) && lane_id() == 0) atomicOr(a.status, R3_DATA_NONFINITE);
}

// One work-group: the loss and its parts.
template <int NT> __device__ void policy_finish(const Policy &a) {
    __shared__ double room[NT / kWave];
    double v[kPolicySums];
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) {
        double s = 0.0;
        for (int p = threadIdx.x; p < a.npieces; p += NT) s += a.part[(int64_t)p * kPolicySums + i];
        v[i] = block_sum<NT>(s, room);
    }
    if (threadIdx.x == 0) {
        const double live = a.tot->live, some = live > 0.0 ? live : 1.0, unit = a.scale != 0.0f ? 1.0 / a.scale : 0.0;
        a.stats[0] = (float)(v[0] + (double)a.kl * v[1] - (double)a.ent * v[2]);
        a.stats[1] = (float)v[0];
        a.stats[2] = (float)(v[1] * unit);
        a.stats[3] = (float)(v[2] * unit);
        a.stats[4] = (float)(v[3] / some);
        a.stats[5] = (float)(v[4] / some);
        a.stats[6] = (float)live;
        a.stats[7] = (float)a.tot->seqs;
    }
}

__global__ void __launch_bounds__(kThreads) policy_segments_kernel(Policy a) { policy_segments<kThreads>(a, blockIdx.x); }
__global__ void __launch_bounds__(1024) policy_sequences_kernel(Policy a) { policy_sequences<1024>(a); }
__global__ void __launch_bounds__(kThreads) policy_tokens_kernel(Policy a) { policy_tokens<kThreads>(a, blockIdx.x); }
__global__ void __launch_bounds__(kThreads) policy_finish_kernel(Policy a) { policy_finish<kThreads>(a); }

struct PolicyPlan {
    int piece, npieces;
    size_t seg, seq, tot, part, total;
};
PolicyPlan policy_plan(int64_t n, int nseq) {
    PolicyPlan p;
    // at least two tokens to a thread, and at most 1024 work-groups until a piece has 8192
    int64_t piece = align_up((size_t)((n + 1023) / 1024), kThreads);
    p.piece = (int)std::min<int64_t>(std::max<int64_t>(piece, 2 * kThreads), 8192);
    p.npieces = (int)((n + p.piece - 1) / p.piece);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    p.seg = take((size_t)(p.npieces + nseq) * sizeof(SegSum));
    p.seq = take((size_t)nseq * sizeof(SeqOut));
    p.tot = take(sizeof(PolicyTotals));
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
    a.cap = D.weight_cap; a.kl = D.kl_coef; a.ent = D.entropy_coef; a.scale = D.scale;
    a.seg = (SegSum *)(base + p.seg); a.seq = (SeqOut *)(base + p.seq); a.tot = (PolicyTotals *)(base + p.tot); a.part = (double *)(base + p.part);
    if (p.npieces) policy_segments_kernel<<<p.npieces, kThreads, 0, s>>>(a);
    policy_sequences_kernel<<<1, 1024, 0, s>>>(a);
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
// probabilities give its part of the loss and its gradient at once.  HBM-bound.
// ---------------------------------------------------------------------------------------------------------------------------------

struct Balance {
    Seqs q;
    int T, E, K;
    int piece0, npieces0;      // of the counts
    int piece, npieces;        // of the logits
    const void *idx;
    int64_t stride;            // of a token's record
    const float *logits;
    int64_t ld, ldd;
    float alpha, zeta;
    int32_t *counts;           // [groups, E]
    float *probs, *stats, *dlogits;
    int32_t *status;
    int32_t *hist;             // [segments of pieces0, E]
    float *psum;               // [segments, E]
    double *lsum;              // [segments][2]: sums of f p and lse^2
    double *tot;               // groups that hold tokens, tokens
};

template <typename IdxT> __device__ void balance_counts(const Balance &a, int p, int *hist) {
    const int64_t lo = (int64_t)p * a.piece0, hi = lesser(lo + a.piece0, a.T);
    if (lo >= hi) return;
    int q0 = a.q.of(lo), q1 = a.q.of(hi - 1);
    q0 = q0 < 0 ? 0 : q0;
    q1 = q1 >= a.q.nseq ? a.q.nseq - 1 : q1;
    bool bad = false;
    for (int q = q0; q <= q1; ++q) {
        const int64_t b = larger(lo, a.q.first(q)), e = lesser(hi, a.q.first(q + 1));
        if (b >= e) continue;
        for (int i = threadIdx.x; i < a.E; i += blockDim.x) hist[i] = 0;
        __syncthreads();
        const IdxT *idx = (const IdxT *)a.idx + b * a.stride;
        const int n = (int)(e - b) * a.K;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int t = i / a.K, id = idx[(int64_t)t * a.stride + (i - t * a.K)];
            if (id < a.E) atomicAdd(&hist[id], 1);
            else bad = true;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.E; i += blockDim.x) a.hist[(int64_t)(p + q) * a.E + i] = hist[i];
        __syncthreads();
    }
    if (a.status && bad) atomicOr(a.status, R3_DATA_IDX_RANGE);
}

template <typename IdxT> __global__ void __launch_bounds__(1024) balance_counts_kernel(Balance a) {
    __shared__ int hist[kMaxE];
    balance_counts<IdxT>(a, blockIdx.x, hist);
}

// counts over a group's segments, a thread to a count; the first work-group also counts groups and tokens
__global__ void __launch_bounds__(kThreads) balance_join_kernel(Balance a) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i < (int64_t)a.q.nseq * a.E) {
        const int q = (int)(i / a.E), e = (int)(i - (int64_t)q * a.E);
        const int64_t b = a.q.first(q), end = a.q.first(q + 1);
        int c = 0;
        if (b < end) {
            const int p0 = (int)(b / a.piece0), p1 = (int)((end - 1) / a.piece0);
            const int32_t *h = a.hist + (int64_t)(p0 + q) * a.E + e;
            int p = p0;
            for (; p + 7 <= p1; p += 8, h += 8 * (int64_t)a.E) {
                int v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = h[u * (int64_t)a.E];
#pragma unroll
                for (int u = 0; u < 8; ++u) c += v[u];
            }
            for (; p <= p1; ++p, h += a.E) c += *h;
        }
        a.counts[i] = c;
    }
    if (blockIdx.x == 0) {
        __shared__ double room[kThreads / kWave];
        double some = 0.0;
        for (int q = threadIdx.x; q < a.q.nseq; q += kThreads) some += a.q.first(q) < a.q.first(q + 1);
        some = block_sum<kThreads>(some, room);
        if (threadIdx.x == 0) {
            a.tot[0] = some;
            a.tot[1] = (double)(a.q.first(a.q.nseq) - a.q.first(0));
        }
    }
}

template <int L, class F> __device__ __forceinline__ float over_lanes(float v, F f) {   // L neighbouring lanes
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, kWave));
    return v;
}

// A token to L lanes, V vectors of four logits to a lane.  Lane l of them has columns 4 (l + L v) .. + 3.
template <int L, int V> __global__ void __launch_bounds__(kThreads) balance_tokens_kernel(Balance a) {
    constexpr int kTok = kThreads / L;       // tokens at a time
    __shared__ float sums[kTok][L * 4];
    __shared__ double room[kThreads / kWave];
    const int64_t lo = (int64_t)blockIdx.x * a.piece, hi = lesser(lo + a.piece, a.T);
    const int l = threadIdx.x % L, w = threadIdx.x / L;
    const int qa = a.q.of(lo), qb = a.q.of(hi - 1);
    bool bad = false;
    auto columns = [&](int v) { const int c = 4 * (l + L * v); return c + 4 <= a.E ? 4 : a.E - c; };   // (none: 0 or less)
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
        float f[V][4], acc[V][4];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                f[v][u] = u < columns(v) ? (float)a.counts[(int64_t)q * a.E + 4 * (l + L * v) + u] * share : 0.0f;
                acc[v][u] = 0.0f;
            }
        double sf = 0.0, sz = 0.0;
        for (int64_t t = b + w; t < e; t += kTok) {
            const float *z = a.logits + t * a.ld;
            float x[V][4];
            float m = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int n = columns(v), c = 4 * (l + L * v);
                if (n == 4) Row<float>::unpack(Row<float>::load(z + c), x[v]);
                else {
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[v][u] = u < n ? z[c + u] : -INFINITY;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) m = __builtin_elementwise_maximum(m, x[v][u]);
            }
            m = over_lanes<L>(m, [](float p, float r) { return __builtin_elementwise_maximum(p, r); });
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
            S = over_lanes<L>(S, [](float p, float r) { return p + r; });
            dot = over_lanes<L>(dot, [](float p, float r) { return p + r; });
            const float inv = empty ? 0.0f : 1.0f / S, mean = dot * inv, lse = empty ? 0.0f : m + logf(S), zg = gz * lse;
            bad |= !isfinite(mean) || !isfinite(lse);
            if (l == 0) {
                sf += mean;
                sz += (double)lse * lse;
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
                    if (n == 4) Row<float>::store(g + c, d);
                    else
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (u < n) g[c + u] = d[u];
                }
            }
        }
        const int64_t seg = (int64_t)blockIdx.x + q;
        sf = block_sum<kThreads>(sf, room);
        sz = block_sum<kThreads>(sz, room);
        if (threadIdx.x == 0) {
            a.lsum[2 * seg] = sf;
            a.lsum[2 * seg + 1] = sz;
        }
        if (a.probs) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int u = 0; u < 4; ++u) sums[w][4 * l + u] = acc[v][u];
                __syncthreads();
                const int c = threadIdx.x, at = 4 * L * v + c;
                if (c < 4 * L && at < a.E) {
                    float s = 0.0f;
                    for (int i = 0; i < kTok; ++i) s += sums[i][c];
                    a.psum[seg * a.E + at] = s;
                }
                __syncthreads();
            }
        }
    }
    if (a.status && __any(bad) && lane_id() == 0) atomicOr(a.status, R3_DATA_NONFINITE);
}

// the first work-group: the loss; the others: mean probabilities, a thread to one
__global__ void __launch_bounds__(kThreads) balance_finish_kernel(Balance a) {
    if (blockIdx.x > 0) {
        const int64_t i = (int64_t)(blockIdx.x - 1) * kThreads + threadIdx.x;
        if (i >= (int64_t)a.q.nseq * a.E) return;
        const int q = (int)(i / a.E), c = (int)(i - (int64_t)q * a.E);
        const int64_t b = a.q.first(q), e = a.q.first(q + 1);
        double s = 0.0;
        if (b < e) {
            const int p0 = (int)(b / a.piece), p1 = (int)((e - 1) / a.piece);
            const float *at = a.psum + (int64_t)(p0 + q) * a.E + c;
            int p = p0;
            for (; p + 7 <= p1; p += 8, at += 8 * (int64_t)a.E) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = at[u * (int64_t)a.E];
#pragma unroll
                for (int u = 0; u < 8; ++u) s += v[u];
            }
            for (; p <= p1; ++p, at += a.E) s += *at;
            s /= (double)(e - b);
        }
        a.probs[i] = (float)s;
        return;
    }
    __shared__ double room[kThreads / kWave];
    double bal = 0.0, z = 0.0;
    // a wave to a group
    for (int q = threadIdx.x / kWave; q < a.q.nseq; q += kThreads / kWave) {
        const int64_t b = a.q.first(q), e = a.q.first(q + 1);
        if (b >= e) continue;
        const int p0 = (int)(b / a.piece), p1 = (int)((e - 1) / a.piece);
        double s = 0.0;
        for (int p = p0 + lane_id(); p <= p1; p += kWave) {
            s += a.lsum[2 * (int64_t)(p + q)];
            z += a.lsum[2 * (int64_t)(p + q) + 1];
        }
        bal += s / (double)(e - b);
    }
    bal = block_sum<kThreads>(bal, room);
    z = block_sum<kThreads>(z, room);
    if (threadIdx.x == 0) {
        const double some = a.tot[0] > 0.0 ? a.tot[0] : 1.0, n = a.tot[1] > 0.0 ? a.tot[1] : 1.0;
        a.stats[0] = (float)((double)a.alpha * bal / some + (double)a.zeta * z / n);
        a.stats[1] = (float)(bal / some);
        a.stats[2] = (float)(z / n);
    }
}

struct BalancePlan {
    int piece0, npieces0, piece, npieces;
    size_t hist, psum, lsum, tot, counts, total;
};
BalancePlan balance_plan(int64_t T, int E, int nseq) {
    BalancePlan p;
    // counts: at most 64 work-groups of 1024 threads, so that few parts are added up
    p.piece0 = (int)std::max<int64_t>((T + 63) / 64, 128);
    p.npieces0 = (int)((T + p.piece0 - 1) / p.piece0);
    const int64_t least = std::max<int64_t>(4, 8192 / E);     // 32 KB of logits
    p.piece = (int)std::max<int64_t>((T + 2047) / 2048, least);
    p.npieces = (int)((T + p.piece - 1) / p.piece);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    p.hist = take((size_t)(p.npieces0 + nseq) * E * sizeof(int32_t));
    p.psum = take((size_t)(p.npieces + nseq) * E * sizeof(float));
    p.lsum = take((size_t)(p.npieces + nseq) * 2 * sizeof(double));
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
    a.piece0 = p.piece0; a.npieces0 = p.npieces0; a.piece = p.piece; a.npieces = p.npieces;
    a.idx = idx; a.stride = stride; a.logits = logits; a.ld = ld; a.ldd = ldd; a.alpha = alpha; a.zeta = zeta;
    a.counts = counts ? counts : (int32_t *)(base + p.counts);
    a.probs = probs; a.stats = stats; a.dlogits = dlogits; a.status = status;
    a.hist = (int32_t *)(base + p.hist); a.psum = (float *)(base + p.psum); a.lsum = (double *)(base + p.lsum); a.tot = (double *)(base + p.tot);
    if (idx_dtype == R3_IDX_U8) balance_counts_kernel<uint8_t><<<p.npieces0, 1024, 0, s>>>(a);
    else balance_counts_kernel<uint16_t><<<p.npieces0, 1024, 0, s>>>(a);
    const unsigned each = (unsigned)(((int64_t)nseq * E + kThreads - 1) / kThreads);
    balance_join_kernel<<<each, kThreads, 0, s>>>(a);
    const int vecs = (E + 3) / 4;
    auto go = [&](auto lanes, auto v) { balance_tokens_kernel<decltype(lanes)::value, decltype(v)::value><<<p.npieces, kThreads, 0, s>>>(a); };
    typedef std::integral_constant<int, 1> one;
    if (vecs <= 2) go(std::integral_constant<int, 2>{}, one{});
    else if (vecs <= 4) go(std::integral_constant<int, 4>{}, one{});
    else if (vecs <= 8) go(std::integral_constant<int, 8>{}, one{});
    else if (vecs <= 16) go(std::integral_constant<int, 16>{}, one{});
    else if (vecs <= 32) go(std::integral_constant<int, 32>{}, one{});
    else if (vecs <= 64) go(std::integral_constant<int, 64>{}, one{});
    else if (vecs <= 128) go(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    else if (vecs <= 256) go(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
    else if (vecs <= 512) go(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
    balance_finish_kernel<<<1 + (probs ? each : 0), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace r3
