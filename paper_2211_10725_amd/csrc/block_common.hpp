// Helpers of the selective leaky block's kernels (selscan.hip, shortconv.hip,
// layer_norm.hip).
#pragma once

#include "snn_internal.hpp"

namespace snn {
namespace {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// V consecutive values of a row as they lie in memory, of any element alignment; only
// the first m are in the row and read, the others are 0.
template <typename T, int V>
struct Raw {
    static constexpr int kWords = V * (int)sizeof(T) / 4, kEach = 4 / (int)sizeof(T);
    static_assert(kWords * 4 == V * (int)sizeof(T), "whole words");
    uint32_t w[kWords];
    __device__ inline void load(const T *p, int m) {
        if (m >= V) {
            __builtin_memcpy(w, p, sizeof(w));
        } else {
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                T t[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    t[j] = k * kEach + j < m ? p[k * kEach + j] : (T)0.f;
                __builtin_memcpy(&w[k], t, 4);
            }
        }
    }
    __device__ inline void get(float (&x)[V]) const {
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            T t[kEach];
            __builtin_memcpy(t, &w[k], 4);
#pragma unroll
            for (int j = 0; j < kEach; ++j) x[k * kEach + j] = (float)t[j];
        }
    }
};

template <typename T, int V>
__device__ inline void load_run(const T *p, int m, float (&v)[V]) {
    Raw<T, V> r;
    r.load(p, m);
    r.get(v);
}

template <typename T, int V>
__device__ inline void store_run(T *p, int m, const float (&v)[V]) {
    if (m >= V) {
        T t[V];
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = (T)v[j];
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < m) p[j] = (T)v[j];
    }
}

// e^x, within e^-150 .. e^88.5 (past that 1 + e^x is 1, or its reciprocal as good as
// nothing).  FINE: to about 1e-7 of itself, 2^p e^(x - p ln 2) with p = fl(x log2 e);
// else with p's error, |x| 2^-24 of itself: for gates of 16-bit tensors, whose outputs of
// 16 bits do not show it and whose sums of gradients in 32 bits have it in each term.
template <bool FINE>
__device__ inline float exp_of(float x) {
    if (!FINE) return __builtin_amdgcn_exp2f(fminf(x * kLog2e, 127.f));
    x = __builtin_amdgcn_fmed3f(x, -150.f, 88.5f);
    const float p = x * kLog2e, e = __builtin_amdgcn_exp2f(p);
    return __builtin_fmaf(e, __builtin_fmaf(p, -kLn2, x), e);
}

// silu and its slope p (1 + z (1 - p)), where 1 - p is taken as e^-z p, which keeps its
// digits while the gate is open.
template <bool FINE>
__device__ inline float silu(float z) {
    return z * __builtin_amdgcn_rcpf(1.f + exp_of<FINE>(-z));
}
template <bool FINE>
__device__ inline void silu_slope(float z, float &act, float &slope) {
    const float e = exp_of<FINE>(-z), p = __builtin_amdgcn_rcpf(1.f + e);
    act = z * p;
    slope = __builtin_fmaf(z, p * (e * p), p);
}

// softplus log(1 + e^x) = max(x, 0) + log1p(e^-|x|) and its slope, the sigmoid.
// log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by the series in s^2 to s^15 (the
// next term is at most 2^-29.5 of the sum): good to the last digits where e is small, as
// the logarithm of a rounded 1 + e is not.  Fine always: states of 32 bits come of it.
__device__ inline void softplus(float x, float &value, float &slope) {
    const float e = exp_of<true>(-__builtin_fabsf(x));
    const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
    float t = 1.f / 15.f;
    t = __builtin_fmaf(t, q, 1.f / 13.f);
    t = __builtin_fmaf(t, q, 1.f / 11.f);
    t = __builtin_fmaf(t, q, 1.f / 9.f);
    t = __builtin_fmaf(t, q, 1.f / 7.f);
    t = __builtin_fmaf(t, q, 1.f / 5.f);
    t = __builtin_fmaf(t, q, 1.f / 3.f);
    value = __builtin_fmaf(2.f, __builtin_fmaf(s * q, t, s), x < 0.f ? 0.f : x);
    const float p = __builtin_amdgcn_rcpf(1.f + e);
    slope = x >= 0.f ? p : e * p;
}

}  // namespace
}  // namespace snn
