// Gradients of the weighted combination and of the dispatch, each as a call of its own, for experts that are not this
// library's:
//   y_t = sum_j g_tj Yp[r_tj]:   dYp[r_tj] = g_tj dy_t,  dg_tj = <dy_t, Yp[r_tj]>,
//                                dz_tj = g_tj (dg_tj - sum_i g_ti dg_ti)   (the gates are a softmax of the selected logits)
//   Xp[r_tj] = x_t:              dx_t = sum_j dXp[r_tj]  (+ add_t)
// Both move rows and compute next to nothing: HBM-bound.
#include "r3_kernels.h"
#include "r3_vec.h"

namespace r3 {
namespace {

// A row of d elements: nvec whole vectors, then rest single elements.  `once`: the rows are marked as read once (non-temporal).
// That is for rows of whole vectors (others share their lines: 30000 x 5 of 501 bf16, sums of rows, marked | not, 50 us | 43) and
// for more of them than half of the 256 MB cache may still hold from whoever wrote them.  marked | not, T x 8 rows of 2048 bf16,
// 33.5 MB for 1024 tokens: combine's gradient T = 1024 14.7 | 13.0 us, 3000 40.0 | 32.7, 4096 52.1 | 51.0, 8192 98.1 | 105.5;
// permute's 3000 20.6 | 17.9, 4096 27.1 | 26.4, 6000 39.4 | 45.2, 16000 100 | 117.
struct Width {
    int d, nvec, rest;
    bool once;
};
template <typename T> Width width(int d, int64_t rows) {
    constexpr int N = Row<T>::kVec;
    return {d, d / N, d % N, d % N == 0 && rows * d * (int64_t)sizeof(T) > 128 << 20};
}
template <bool ONCE, typename T> __device__ __forceinline__ typename Row<T>::V load_row(const T *p) {
    if constexpr (ONCE) return Row<T>::load_once(p);
    else return Row<T>::load(p);
}

struct CombineBwd {
    int T, K;
    int64_t S;
    Width w;
    const void *dy, *Yp;
    const float *gates;
    const int32_t *inv_perm;
    void *dYp;
    float *dgates, *dz;
};

// W waves to the columns of a token's rows, a vector of 16 bytes to a lane at a time, times P waves to its slots, G slots at a
// time.  Two rows a wave and two waves to the slots: with more rows in one wave the loads and stores of fewer, longer waves move
// less (65536 x 8 of 2048 bf16, 8 x 1 | 4 x 2 | 2 x 4 | 2 x 2: 898 | 884 | 886 | 882 us; 30000 x 6 of 1000 178 | 176 | 173 | 172;
// 30000 x 5 of 501 103 | 105 | 97 | 92; 30000 x 4 of 1024 f32 204 | 217 | 226 | 183), and the dot products of a token meet once,
// in LDS.  dYp may be Yp: an element is read and written by one thread.
template <typename T, int G, int W, int P, bool ONCE>
__global__ void __launch_bounds__(W * P > 4 ? W * P * kWave : 256)
combine_backward_kernel(CombineBwd a) {
    typedef Row<T> R;
    constexpr int N = R::kVec;
    constexpr int kTok = W * P < 4 ? 4 / (W * P) : 1;   // tokens of a work-group
    __shared__ float part[kTok * W * P][kMaxK];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
    const int t = blockIdx.x * kTok + wave / (W * P);
    const bool some = t < a.T;   // (waves of the last work-group may have no token, and still meet the others)
    if (W * P == 1 && !some) return;
    const int first_slot = wave / W % P * G, first = wave % W * kWave + lane;
    const T *dy = (const T *)a.dy + (int64_t)t * a.w.d;
    const int32_t *rows = a.inv_perm + (int64_t)t * a.K;
    const float *gates = a.gates + (int64_t)t * a.K;
    const bool dots = a.Yp != nullptr;
    float mine = 0.0f;   // lane j: the dot product of slot j over this wave's columns
    for (int j0 = some ? first_slot : a.K; j0 < a.K; j0 += G * P) {
        int64_t at[G];
        float g[G], dot[G];
        bool in[G];
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const int32_t r = j0 + j < a.K ? rows[j0 + j] : -1;
            in[j] = r >= 0 && r < a.S;
            at[j] = in[j] ? (int64_t)r * a.w.d : 0;
            g[j] = j0 + j < a.K ? gates[j0 + j] : 0.0f;
            dot[j] = 0.0f;
        }
        for (int c = first; c < a.w.nvec; c += W * kWave) {
            float x[N];
            typename R::V v[G];
            R::unpack(R::load(dy + c * N), x);
            if (dots) {
#pragma unroll
                for (int j = 0; j < G; ++j) v[j] = load_row<ONCE>((const T *)a.Yp + at[j] + c * N);
            }
#pragma unroll
            for (int j = 0; j < G; ++j) {
                if (dots) {
                    float y[N];
                    R::unpack(v[j], y);
#pragma unroll
                    for (int u = 0; u < N; ++u) dot[j] = fmaf(x[u], y[u], dot[j]);
                }
                if (a.dYp && in[j]) {
                    float o[N];
#pragma unroll
                    for (int u = 0; u < N; ++u) o[u] = g[j] * x[u];
                    R::store_once((T *)a.dYp + at[j] + c * N, o);
                }
            }
        }
        if (first < a.w.rest) {
            const int e = a.w.nvec * N + first;
            const float x = Elem<T>::ld(dy + e);
#pragma unroll
            for (int j = 0; j < G; ++j) {
                if (dots) dot[j] = fmaf(x, Elem<T>::ld((const T *)a.Yp + at[j] + e), dot[j]);
                if (a.dYp && in[j]) Elem<T>::st((T *)a.dYp + at[j] + e, g[j] * x);
            }
        }
        if (dots) {
#pragma unroll
            for (int j = 0; j < G; ++j) {
                const float s = wave_total(in[j] ? dot[j] : 0.0f);
                if (lane == j0 + j) mine = s;
            }
        }
    }
    if (!dots) return;
    if constexpr (W * P > 1) {
        part[wave][lane] = mine;
        __syncthreads();
        if (wave % (W * P) > 0 || !some) return;
        mine = 0.0f;
#pragma unroll
        for (int i = 0; i < W * P; ++i) mine += part[wave + i][lane];
    }
    const float g = lane < a.K ? gates[lane] : 0.0f;
    const float mix = wave_total(lane < a.K ? g * mine : 0.0f);
    if (lane < a.K) {
        if (a.dgates) a.dgates[(int64_t)t * a.K + lane] = mine;
        if (a.dz) a.dz[(int64_t)t * a.K + lane] = g * (mine - mix);
    }
}

struct PermuteBwd {
    int T, K;
    uint32_t chunks;   // of 64 vectors, in a row
    int64_t S;
    Width w;
    const void *dXp, *add;
    const int32_t *inv_perm;
    void *dx;
};

// A wave to 64 vectors of a token's row, the last one of a row to the elements behind them too.  Two rows at a time: with all
// K on their way at once 65536 x 8 of 2048 bf16 take 488 us, four at a time 484, two 476; 30000 x 6 of 1000 82 | 82 | 77 (many
// waves keep enough loads on their way).  dx may be add.
template <typename T, int G, bool ONCE>
__global__ void __launch_bounds__(256)
permute_backward_kernel(PermuteBwd a) {
    typedef Row<T> R;
    constexpr int N = R::kVec;
    const uint32_t item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), t = item / a.chunks;
    if (t >= (uint32_t)a.T) return;
    const int chunk = item - t * a.chunks, c = chunk * kWave + lane_id();
    const int32_t *rows = a.inv_perm + (int64_t)t * a.K;
    const T *dXp = (const T *)a.dXp, *add = a.add ? (const T *)a.add + (int64_t)t * a.w.d : nullptr;
    T *dx = (T *)a.dx + (int64_t)t * a.w.d;
    if (c < a.w.nvec) {
        float acc[N] = {};
        if (add) R::unpack(R::load(add + c * N), acc);
        for (int j0 = 0; j0 < a.K; j0 += G) {
            typename R::V v[G];
            bool in[G];
#pragma unroll
            for (int j = 0; j < G; ++j) {
                const int32_t r = j0 + j < a.K ? rows[j0 + j] : -1;
                in[j] = r >= 0 && r < a.S;
                v[j] = load_row<ONCE>(dXp + (in[j] ? (int64_t)r * a.w.d : 0) + c * N);
            }
#pragma unroll
            for (int j = 0; j < G; ++j) {
                float f[N];
                R::unpack(v[j], f);
                if (in[j]) {
#pragma unroll
                    for (int u = 0; u < N; ++u) acc[u] += f[u];
                }
            }
        }
        R::store(dx + c * N, acc);
    }
    if (chunk == (int)a.chunks - 1 && lane_id() < a.w.rest) {
        const int e = a.w.nvec * N + lane_id();
        float acc = add ? Elem<T>::ld(add + e) : 0.0f;
        for (int j = 0; j < a.K; ++j) {
            const int32_t r = rows[j];
            if (r >= 0 && r < a.S) acc += Elem<T>::ld(dXp + (int64_t)r * a.w.d + e);
        }
        Elem<T>::st(dx + e, acc);
    }
}

}  // namespace

bool route_backward_supported(int T, int d, int act) {
    const int per = 1024 / (act == R3_BF16 ? 2 : 4);   // elements of 64 vectors
    return (int64_t)T * (((int64_t)d + per - 1) / per) <= 1 << 24;   // a token takes 512 threads at most
}

hipError_t launch_combine_backward(int T, int d, int K, int act, const void *dy, const void *Yp, const float *gates, const int32_t *inv_perm,
                                   void *dYp, float *dgates, float *dz, hipStream_t s) {
    ProfScope ps(PROF_COMBINE_BWD, s);
    CombineBwd a = {T, K, (int64_t)T * K, {}, dy, dgates || dz ? Yp : nullptr, gates, inv_perm, dYp, dgates, dz};
    auto go = [&](auto type) {
        typedef decltype(type) E;
        a.w = width<E>(d, a.S);
        auto launch = [&](auto g, auto w, auto p) {
            constexpr int G = decltype(g)::value, W = decltype(w)::value, P = decltype(p)::value, kTok = W * P < 4 ? 4 / (W * P) : 1;
            auto k = a.w.once ? combine_backward_kernel<E, G, W, P, true> : combine_backward_kernel<E, G, W, P, false>;
            k<<<(T + kTok - 1) / kTok, kTok * W * P * kWave, 0, s>>>(a);
        };
        auto by_width = [&](auto g, auto p) {
            if (a.w.nvec <= kWave) launch(g, std::integral_constant<int, 1>{}, p);
            else if (a.w.nvec <= 2 * kWave) launch(g, std::integral_constant<int, 2>{}, p);
            else launch(g, std::integral_constant<int, 4>{}, p);
        };
        if (K == 1) by_width(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
        else by_width(std::integral_constant<int, 2>{}, std::integral_constant<int, 2>{});
    };
    if (act == R3_BF16) go(bf16_t{});
    else go(float{});
    return hipGetLastError();
}

hipError_t launch_permute_backward(int T, int d, int K, int act, const void *dXp, const int32_t *inv_perm, const void *add, void *dx,
                                   hipStream_t s) {
    ProfScope ps(PROF_PERMUTE_BWD, s);
    PermuteBwd a = {T, K, 1, (int64_t)T * K, {}, dXp, add, inv_perm, dx};
    auto go = [&](auto type) {
        typedef decltype(type) E;
        a.w = width<E>(d, a.S);
        a.chunks = a.w.nvec > 0 ? (a.w.nvec + kWave - 1) / kWave : 1;
        const unsigned blocks = (unsigned)(((int64_t)T * a.chunks + 3) / 4);
        auto k = K == 1 ? (a.w.once ? permute_backward_kernel<E, 1, true> : permute_backward_kernel<E, 1, false>)
                        : (a.w.once ? permute_backward_kernel<E, 2, true> : permute_backward_kernel<E, 2, false>);
        k<<<blocks, 256, 0, s>>>(a);
    };
    if (act == R3_BF16) go(bf16_t{});
    else go(float{});
    return hipGetLastError();
}

}  // namespace r3
