// Rows of elements in loads and stores of 16 bytes at any element's address: rows of odd widths and strides start
// anywhere, and the hardware takes such addresses.  Reductions over a wave.
#pragma once
#include "r3_common.h"

namespace r3 {

template <typename T> struct Row;
template <> struct Row<bf16_t> {
    static constexpr int kVec = 8;
    typedef uint32_t V __attribute__((ext_vector_type(4)));
    typedef V U __attribute__((aligned(2)));
    static __device__ __forceinline__ V load(const bf16_t *p) { return *(const U *)p; }
    static __device__ __forceinline__ V load_once(const bf16_t *p) { return __builtin_nontemporal_load((const U *)p); }
    static __device__ __forceinline__ void unpack(const V &v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ V pack(const float *f) {
        V v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
        return v;
    }
    static __device__ __forceinline__ void store(bf16_t *p, const float *f) { *(U *)p = pack(f); }
    static __device__ __forceinline__ void store_once(bf16_t *p, const float *f) { __builtin_nontemporal_store(pack(f), (U *)p); }
};
template <> struct Row<float> {
    static constexpr int kVec = 4;
    typedef float V __attribute__((ext_vector_type(4)));
    typedef V U __attribute__((aligned(4)));
    static __device__ __forceinline__ V load(const float *p) { return *(const U *)p; }
    static __device__ __forceinline__ V load_once(const float *p) { return __builtin_nontemporal_load((const U *)p); }
    static __device__ __forceinline__ void unpack(const V &v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = v[i];
    }
    static __device__ __forceinline__ V pack(const float *f) { return V{f[0], f[1], f[2], f[3]}; }
    static __device__ __forceinline__ void store(float *p, const float *f) { *(U *)p = pack(f); }
    static __device__ __forceinline__ void store_once(float *p, const float *f) { __builtin_nontemporal_store(pack(f), (U *)p); }
};

// A value over all 64 lanes, in every lane: six moves within the vector pipe (a row's neighbours 1, 2, 4, 8 on, the last lane
// of a row to the next row, of the first half to the second) instead of six trips through LDS.  `none`: what f leaves alone.
template <int CTRL, int ROWS> __device__ __forceinline__ float lane_move(float v, float none) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <class F> __device__ __forceinline__ float over_wave(float v, float none, F f) {
    v = f(v, lane_move<0x111, 0xf>(v, none));
    v = f(v, lane_move<0x112, 0xf>(v, none));
    v = f(v, lane_move<0x114, 0xf>(v, none));
    v = f(v, lane_move<0x118, 0xf>(v, none));
    v = f(v, lane_move<0x142, 0xa>(v, none));
    v = f(v, lane_move<0x143, 0xc>(v, none));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}
__device__ __forceinline__ float wave_total(float v) {
    return over_wave(v, 0.0f, [](float a, float b) { return a + b; });
}

}  // namespace r3
