// Norms before and after a block with its gate and residual scale, forward and
// backward, and activation checkpoints in 8 bits (include/snn.h, "leaky
// sequence block").
//
// Every call is one pass over HBM: a row stays in registers between its sums
// and the values that need them, as far as the registers go (below).  A row belongs to TPR threads (a wave for
// short rows, else a workgroup), thread t holding the NV runs of 8 channels
// 8 (i TPR + t): one 16-byte access per 16-bit run.  Rows may start on any
// element (odd widths, slices), which the memory pipeline takes as it is; only
// the last run of a row whose width is no multiple of 8 goes value by value.
// Workgroups take rows in turn with the weights in registers, and the
// backward's column sums too: one partial row per workgroup, added in
// workgroup order by a second kernel.
//
// Bound by HBM.  16384 rows of 2048 (bf16 block, fp32 residual stream, 16 heads):
// forward 93 us, 5.0 TB/s, as a large copy; backward 155 to 164, 4.5 to 4.8 TB/s
// (all in bf16 131, 4.1).  8192 rows of 4096 (fp16) with 8-bit checkpoints: 119 and 166.
//
// The backward holds more than four waves of a SIMD have registers for.  With a 16-bit
// block 9 to 33 registers a lane lie in scratch (17 in the backward above), in fp32 none
// with up to 512 threads, which then take three waves, and 35 or 70 with 1024.  Rows of
// more than 8192 channels, two runs a thread, leave most of theirs there: 4096 rows of
// 12288 there and back take 1233 us in fp32 and 990 with a bf16 block, 1.6 and 1.4 TB/s
// (forward alone 254 and 222, 4.0 and 3.2).
#include <float.h>

#include "snn_internal.hpp"

namespace snn {
namespace {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLo = 1.9259629911266175e-8f;  // log2(e) - kLog2e
constexpr float kLn2 = 0.6931471805599453f;

// e^x = 2^(x log2 e) with the product's rounding error put back (2^x itself is
// good to an ulp): relative error about 1e-7 over the whole range.
__device__ inline float exp_of(float x) {
    const float p = x * kLog2e;
    const float r = __builtin_fmaf(x, kLog2e, -p) + x * kLog2eLo;
    const float e = __builtin_amdgcn_exp2f(p);
    // no correction where the power has left the range (r may be NaN there)
    return e > 0.f && e < __builtin_inff() ? __builtin_fmaf(e, r * kLn2, e) : e;
}

// The gate's factor and its derivative.  The sigmoid's is p (1 - p), taken as p e^-g p:
// 1 - p of an open gate would have few digits of e^-g left, from g = 17 on none.
template <bool SLOPE>
__device__ inline void gate_of(int gate, float g, float &act, float &slope) {
    if (gate == SNN_GATE_MUL) {
        act = g;
        slope = 1.f;
        return;
    }
    const float e = exp_of(-g), p = __builtin_amdgcn_rcpf(1.f + e);
    act = gate == SNN_GATE_SILU ? g * p : p;
    if (SLOPE) {
        const float q = p * (fminf(e, FLT_MAX) * p);  // (p is 0 where e is infinite)
        slope = gate == SNN_GATE_SILU ? __builtin_fmaf(g, q, p) : q;
    }
}

// 8 values from / to memory of any element alignment; `m` of them are in the row
template <typename T>
__device__ inline void load8(const T *p, int m, float (&v)[8]) {
    if (m >= 8) {
        T t[8];
        __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)t[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < m ? (float)p[j] : 0.f;
    }
}
// 16-byte accesses past the caches: the backward's tensors are read and written
// once (16384 rows of 2048 bf16 channels: 174 us through the caches, 155 past
// them; the forward's outputs are soon read again and gain nothing).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

template <int WORDS>
__device__ inline void stream_in(uint32_t (&w)[WORDS], const void *p) {
    if constexpr (WORDS == 2) {
        const u32x2 v = __builtin_nontemporal_load((const u32x2_any *)p);
        w[0] = v[0], w[1] = v[1];
    } else {
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) {
            const u32x4 v = __builtin_nontemporal_load((const u32x4_any *)p + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
        }
    }
}

// the same, kept as they lie in memory until they are needed
template <typename T>
struct Run {
    static constexpr int kWords = 2 * sizeof(T), kEach = 4 / sizeof(T);
    uint32_t w[kWords];
    __device__ inline void load(const T *p, int m) {
        if (m >= 8) {
            stream_in(w, p);
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
    __device__ inline void get(float (&x)[8]) const {
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            T t[kEach];
            __builtin_memcpy(t, &w[k], 4);
#pragma unroll
            for (int j = 0; j < kEach; ++j) x[k * kEach + j] = (float)t[j];
        }
    }
};
template <bool STREAM = false, typename T>
__device__ inline void store8(T *p, int m, const float (&v)[8]) {
    if (m >= 8) {
        T t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = (T)v[j];
        if constexpr (STREAM) {
            u32x4 w[sizeof(t) / 16];
            __builtin_memcpy(w, t, sizeof(t));
#pragma unroll
            for (int i = 0; i < (int)(sizeof(t) / 16); ++i)
                __builtin_nontemporal_store(w[i], (u32x4_any *)p + i);
        } else {
            __builtin_memcpy(p, t, sizeof(t));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < m) p[j] = (T)v[j];
    }
}
__device__ inline void load_weights(const float *w, int64_t e, int m, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 1.f;
    if (w && m > 0) load8(w + e, m, v);
}

template <int TPR, int NV>
__device__ inline void load_row_weights(const GateNorm &a, int (&m)[NV], int64_t (&e)[NV],
                                        float (&cw)[NV][8], float (&wr)[NV][8]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float sc[8];
        e[i] = 8 * (i * TPR + threadIdx.x % TPR);
        m[i] = (int)min((int64_t)8, max((int64_t)0, a.n - e[i]));
        load_weights(a.w_post, e[i], m[i], cw[i]);
        load_weights(a.scale, e[i], m[i], sc);
        load_weights(a.w_pre, e[i], m[i], wr[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) cw[i][j] *= sc[j];
    }
}

// ---- 8-bit checkpoints: `lanes` consecutive lanes (1 .. 16) hold a block of values --
constexpr float kMinMax = 0x1p-100f;

__device__ inline void encode8(const float (&v)[8], int8_t *code, float *scale, int m,
                               int lanes) {
    uint32_t top = 0;  // |x| as bits: NaN above infinity above every number
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    for (int off = 1; off < lanes; off <<= 1)
        top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
    const float t = __uint_as_float(top);
    const bool fine = top < 0x7f800000u, some = fine && t >= kMinMax;
    const float up = some ? 127.f / t : 0.f;
    int8_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = some ? (int8_t)__builtin_rintf(v[j] * up) : (int8_t)0;
    if (m >= 8) {
        __builtin_memcpy(code, c, 8);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < m) code[j] = c[j];
    }
    if ((threadIdx.x & (lanes - 1)) == 0 && m > 0)
        *scale = !fine ? __builtin_nanf("") : some ? t * (float)(1.0 / 127.0) : 0.f;
}
__device__ inline void decode8(const int8_t *code, float scale, int m, float (&v)[8]) {
    int8_t c[8] = {};
    if (m >= 8) {
        __builtin_memcpy(c, code, 8);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < m) c[j] = code[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)c[j] * scale;
}

// ---- sums over a row -------------------------------------------------------------
// Sum over the TPR threads of a row (fixed order); `red` holds a slot per wave.
template <int TPR, int N>
__device__ inline void row_sum(float (&s)[N], float *red) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) s[k] += __shfl_xor(s[k], off, 64);
    if (TPR > 64) {
        const int w = threadIdx.x % TPR >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) red[w * N + k] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            s[k] = red[k];
            for (int i = 1; i < TPR / 64; ++i) s[k] += red[i * N + k];
        }
        __syncthreads();
    }
}

// Sum of s over the groups of the row: on entry s[i] is the sum over run i of
// this thread, on return that of the run's whole group.  `gl` runs make a group
// (0: the row is one group).  A power of two up to a wave adds by exchanges,
// anything else through `vec` (one slot per run of the row), where each thread adds
// its whole group: right for any count, and slow for large groups (8192 rows there and
// back, bf16 block: four groups of 1000 475 us, one group of 4000 297; four of 2048
// 1427 against 603; two of 8192 9638 against 2084).
template <int TPR, int NV>
__device__ inline void group_sum(float (&s)[NV], int gl, int runs, float *red, float *vec) {
    if (gl == 0) {
        float t[1] = {s[0]};
#pragma unroll
        for (int i = 1; i < NV; ++i) t[0] += s[i];
        row_sum<TPR, 1>(t, red);
#pragma unroll
        for (int i = 0; i < NV; ++i) s[i] = t[0];
    } else if (gl <= 64 && (gl & (gl - 1)) == 0) {
        for (int off = 1; off < gl; off <<= 1)
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] += __shfl_xor(s[i], off, 64);
    } else {
        const int t = threadIdx.x % TPR;
#pragma unroll
        for (int i = 0; i < NV; ++i) vec[i * TPR + t] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int r = i * TPR + t;
            float a = 0.f;
            if (r < runs)
                for (int k = r / gl * gl, e = k + gl; k < e; ++k) a += vec[k];
            s[i] = a;
        }
        __syncthreads();
    }
}

template <int TPR>
constexpr int block_threads() { return TPR > 256 ? TPR : 256; }

template <typename XT, typename YT, int TPR, int NV>
__global__ __launch_bounds__(block_threads<TPR>()) void gate_norm_fwd_kernel(GateNormFwd c) {
    constexpr int RPB = block_threads<TPR>() / TPR;
    __shared__ float red[RPB][16];
    __shared__ float vec[RPB][TPR * NV];
    const int slot = threadIdx.x / TPR;
    const GateNorm a = c.a;
    const int runs = (a.n + 7) / 8, gl = a.groups == 1 ? 0 : a.n / a.groups / 8;
    const float inv_n = 1.f / (float)a.n, inv_d = 1.f / (float)(a.n / a.groups);
    int m[NV];
    int64_t e[NV];
    float cw[NV][8], wr[NV][8];  // w_post scale, w_pre
    load_row_weights<TPR, NV>(a, m, e, cw, wr);
    const int64_t step = (int64_t)gridDim.x * RPB, nb = ckpt_blocks(a.n, a.block);
    // every thread of the workgroup takes part in each round's barriers
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step) {
        const int64_t row = r0 + slot;
        const bool live = row < a.rows;
        const XT *x = static_cast<const XT *>(c.x) + row * a.ld_x;
        float xv[NV][8], yv[NV][8], gv[NV][8], s[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = live ? m[i] : 0;
            load8(x + e[i], k, xv[i]);
            if (c.y) load8(static_cast<const YT *>(c.y) + row * a.ld_y + e[i], k, yv[i]);
            if (c.g) load8(static_cast<const YT *>(c.g) + row * a.ld_g + e[i], k, gv[i]);
        }
        if (c.y) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) s[i] = __builtin_fmaf(yv[i][j], yv[i][j], s[i]);
            }
            group_sum<TPR, NV>(s, gl, runs, red[slot], vec[slot]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int k = live ? m[i] : 0;
                const float ry = 1.f / __builtin_sqrtf(__builtin_fmaf(s[i], inv_d, a.eps));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float act = 1.f, slope;
                    if (c.g) gate_of<false>(a.gate, gv[i][j], act, slope);
                    xv[i][j] += yv[i][j] * ry * act * cw[i][j];
                }
                store8(static_cast<XT *>(c.x_out) + row * a.ld_x + e[i], k, xv[i]);
                const int64_t blk = row * nb + e[i] / a.block;
                if (c.y8) encode8(yv[i], c.y8 + row * a.n + e[i], c.y8s + blk, k, a.block / 8);
                if (c.g8) encode8(gv[i], c.g8 + row * a.n + e[i], c.g8s + blk, k, a.block / 8);
            }
        }
        if (!c.h) continue;
        float q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                q[0] = __builtin_fmaf(xv[i][j], xv[i][j], q[0]);
        row_sum<TPR, 1>(q, red[slot]);
        const float rx = 1.f / __builtin_sqrtf(__builtin_fmaf(q[0], inv_n, a.eps));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) xv[i][j] *= rx * wr[i][j];
            store8(static_cast<YT *>(c.h) + row * a.ld_h + e[i], live ? m[i] : 0, xv[i]);
        }
    }
}

template <typename XT, typename YT, bool CKPT, int TPR, int NV>
__global__ __launch_bounds__(block_threads<TPR>(), sizeof(YT) == 2 || TPR == 1024 ? 4 : 3) void
gate_norm_bwd_kernel(GateNormBwd c) {
    constexpr int RPB = block_threads<TPR>() / TPR;
    __shared__ float red[RPB][32];
    __shared__ float vec[RPB][TPR * NV];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const GateNorm a = c.a;
    const int runs = (a.n + 7) / 8, gl = a.groups == 1 ? 0 : a.n / a.groups / 8;
    const float inv_n = 1.f / (float)a.n, inv_d = 1.f / (float)(a.n / a.groups);
    const bool block = CKPT || c.y;
    int m[NV];
    int64_t e[NV];
    float cw[NV][8], wr[NV][8];  // w_post scale, w_pre
    load_row_weights<TPR, NV>(a, m, e, cw, wr);
    // sums over this workgroup's rows: of dx act(gate) yhat, which times scale is
    // w_post's gradient and times w_post scale's, and of dh xhat, w_pre's
    float a_post[NV][8] = {}, a_pre[NV][8] = {};
    const int64_t step = (int64_t)gridDim.x * RPB, nb = ckpt_blocks(a.n, a.block);
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step) {
        const int64_t row = r0 + slot;
        const bool live = row < a.rows;
        float dx[NV][8], dh[NV][8], xo[NV][8], yv[NV][8], gv[NV][8], s[NV];
        Run<XT> rdx[NV], rxo[NV];
        Run<YT> rdh[NV], ry_[NV], rg[NV];
        Run<int8_t> cy[NV], cg[NV];
        float sy[NV], sg[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = live ? m[i] : 0;
            const int64_t at = row * a.n + e[i], blk = row * nb + e[i] / a.block;
            rdx[i].load(static_cast<const XT *>(c.dxo) + row * a.ld_x + e[i], c.dxo ? k : 0);
            if (c.dh) {
                rdh[i].load(static_cast<const YT *>(c.dh) + row * a.ld_h + e[i], k);
                rxo[i].load(static_cast<const XT *>(c.xo) + row * a.ld_x + e[i], k);
            }
            if (CKPT) {
                cy[i].load(c.y8 + at, k);
                sy[i] = k > 0 ? c.y8s[blk] : 0.f;
                if (c.g8) {
                    cg[i].load(c.g8 + at, k);
                    sg[i] = k > 0 ? c.g8s[blk] : 0.f;
                }
            } else {
                if (c.y) ry_[i].load(static_cast<const YT *>(c.y) + row * a.ld_y + e[i], k);
                if (c.g) rg[i].load(static_cast<const YT *>(c.g) + row * a.ld_g + e[i], k);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) rdx[i].get(dx[i]);
        if (c.dh) {
            float q[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                rdh[i].get(dh[i]);
                rxo[i].get(xo[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    q[0] = __builtin_fmaf(xo[i][j], xo[i][j], q[0]);
                    q[1] = __builtin_fmaf(xo[i][j], dh[i][j] * wr[i][j], q[1]);
                }
            }
            row_sum<TPR, 2>(q, red[slot]);
            const float rx = 1.f / __builtin_sqrtf(__builtin_fmaf(q[0], inv_n, a.eps));
            const float mean = q[1] * rx * inv_n;  // of xhat dxhat
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float hat = xo[i][j] * rx;
                    dx[i][j] += rx * (dh[i][j] * wr[i][j] - hat * mean);
                    a_pre[i][j] = __builtin_fmaf(dh[i][j], hat, a_pre[i][j]);
                }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            store8<true>(static_cast<XT *>(c.dx) + row * a.ld_x + e[i], live ? m[i] : 0, dx[i]);
        if (!block) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            s[i] = 0.f;
            if (CKPT) {
                cy[i].get(yv[i]);
                if (c.g8) cg[i].get(gv[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) yv[i][j] *= sy[i], gv[i][j] *= sg[i];
            } else {
                ry_[i].get(yv[i]);
                if (c.g) rg[i].get(gv[i]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i] = __builtin_fmaf(yv[i][j], yv[i][j], s[i]);
        }
        group_sum<TPR, NV>(s, gl, runs, red[slot], vec[slot]);
        float ry[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            ry[i] = 1.f / __builtin_sqrtf(__builtin_fmaf(s[i], inv_d, a.eps));
            s[i] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float act = 1.f, slope = 0.f;
                if (a.gate != SNN_GATE_NONE) gate_of<true>(a.gate, gv[i][j], act, slope);
                const float hat = yv[i][j] * ry[i], d = dx[i][j] * cw[i][j];
                a_post[i][j] = __builtin_fmaf(dx[i][j] * act, hat, a_post[i][j]);
                gv[i][j] = d * hat * slope;
                yv[i][j] = hat;
                dx[i][j] = d * act;
                s[i] = __builtin_fmaf(hat, dx[i][j], s[i]);
            }
        }
        group_sum<TPR, NV>(s, gl, runs, red[slot], vec[slot]);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = live ? m[i] : 0;
            const float mean = s[i] * inv_d;
#pragma unroll
            for (int j = 0; j < 8; ++j) yv[i][j] = ry[i] * (dx[i][j] - yv[i][j] * mean);
            store8<true>(static_cast<YT *>(c.dy) + row * a.ld_y + e[i], k, yv[i]);
            if (c.dg) store8<true>(static_cast<YT *>(c.dg) + row * a.ld_g + e[i], k, gv[i]);
        }
    }
    // the workgroup's column sums, its rows' slots added in order
    __shared__ float col[RPB > 1 ? TPR * NV * 8 : 1];
    float(*sums[2])[8] = {a_post, a_pre};
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float *part = c.part + ((int64_t)w * gridDim.x + blockIdx.x) * a.n;
        for (int k = 1; k < RPB; ++k) {
            __syncthreads();
            if (slot == k)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) col[j * TPR * NV + i * TPR + t] = sums[w][i][j];
            __syncthreads();
            if (slot == 0)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sums[w][i][j] += col[j * TPR * NV + i * TPR + t];
        }
        if (slot == 0)
#pragma unroll
            for (int i = 0; i < NV; ++i) store8(part + e[i], m[i], sums[w][i]);
    }
}

// Column sums over the workgroups' partial rows, in order within each of the 16
// waves' shares, then over the waves; w_post's and scale's gradients are the
// first sum times each other.  6.6 us for 1024 workgroups' rows of 1001 (32 workgroups
// of 64 columns), 7.5 of 2048: latency.
__global__ __launch_bounds__(1024) void column_sum_kernel(GateNormBwd c, int blocks) {
    const bool pre = blockIdx.y == 1;
    if (pre ? !c.dw_pre : !c.dw_post && !c.dscale) return;  // the whole workgroup
    __shared__ float sum[16][64];
    const int n = c.a.n;
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane;
    const float *p = c.part + (int64_t)blockIdx.y * blocks * n + col;
    // 16 loads at a time on their way: one after the other they cost 22 us of
    // latency for 1024 workgroups
    float s = 0.f;
    if (col < n)
        for (int b = w; b < blocks; b += 256) {
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = b + 16 * i < blocks ? p[(int64_t)(b + 16 * i) * n] : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) s += x[i];
        }
    sum[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < n) {
        for (int i = 1; i < 16; ++i) s += sum[i][lane];
        if (pre) {
            c.dw_pre[col] = s;
        } else {
            if (c.dw_post) c.dw_post[col] = c.a.scale ? s * c.a.scale[col] : s;
            if (c.dscale) c.dscale[col] = c.a.w_post ? s * c.a.w_post[col] : s;
        }
    }
}

// 16 lanes take 128 values of a row
template <typename T, bool SAVE>
__global__ __launch_bounds__(256) void checkpoint_kernel(int64_t units, uint32_t per_row, int n,
                                                         int block, int64_t ld, T *x,
                                                         int8_t *codes, float *scales) {
    const int64_t u = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 16 + threadIdx.x / 16;
    const bool live = u < units;
    const int64_t row = live ? (uint32_t)u / per_row : 0;
    const int e = live ? (int)((uint32_t)u % per_row) * 128 + 8 * (threadIdx.x & 15) : 0;
    const int m = live ? min(8, max(0, n - e)) : 0;
    const int64_t b = row * ckpt_blocks(n, block) + e / block;
    float v[8];
    if (SAVE) {
        load8(x + row * ld + e, m, v);
        encode8(v, codes + row * n + e, scales + b, m, block / 8);
    } else if (m > 0) {
        decode8(codes + row * n + e, scales[b], m, v);
        store8(x + row * ld + e, m, v);
    }
}

// Threads of a row: the fewest whose runs of 8 cover it, so that a row takes
// one run per thread (of 512 to 1024, two runs of a wave: the backward's
// registers then halve the waves that a CU holds); two only past 8192.
int threads_per_row(int n) {
    int t = 64;
    while (t < 1024 && 8 * t < n) t *= 2;
    return t;
}
int rows_per_block(int n) { return std::max(1, 256 / threads_per_row(n)); }

// Workgroups: four of 256 threads per compute unit, as many as are resident at once
// (16384 rows of 2048 there and back 255 us, with half as many 290, with 1.5 times
// 288) but for the backward of fp32 blocks, of which three are, and one of 512 threads
// where two are launched.  The backward's partial sums are [2][blocks][n].
int row_blocks(int64_t rows, int64_t n) {
    const int64_t rpb = rows_per_block((int)n);
    const int64_t most = 4 * kPlanCus * 256 / std::max(256, threads_per_row((int)n));
    return (int)std::min<int64_t>((rows + rpb - 1) / rpb, most);
}

#define GATE_NORM_SIZES(KERNEL, ...)                                                           \
    if (n <= 512) KERNEL<__VA_ARGS__, 64, 1><<<grid, 256, 0, s>>>(c);                          \
    else if (n <= 1024) KERNEL<__VA_ARGS__, 128, 1><<<grid, 256, 0, s>>>(c);                   \
    else if (n <= 2048) KERNEL<__VA_ARGS__, 256, 1><<<grid, 256, 0, s>>>(c);                   \
    else if (n <= 4096) KERNEL<__VA_ARGS__, 512, 1><<<grid, 512, 0, s>>>(c);                   \
    else if (n <= 8192) KERNEL<__VA_ARGS__, 1024, 1><<<grid, 1024, 0, s>>>(c);                 \
    else KERNEL<__VA_ARGS__, 1024, 2><<<grid, 1024, 0, s>>>(c);

template <typename XT, typename YT>
void run_fwd(const GateNormFwd &c, hipStream_t s) {
    const int n = c.a.n, grid = row_blocks(c.a.rows, n);
    GATE_NORM_SIZES(gate_norm_fwd_kernel, XT, YT)
}

template <typename XT, typename YT>
void run_bwd(const GateNormBwd &c, hipStream_t s) {
    const int n = c.a.n, grid = row_blocks(c.a.rows, n);
    if (grid > 0) {
        if (c.y8) {
            GATE_NORM_SIZES(gate_norm_bwd_kernel, XT, YT, true)
        } else {
            GATE_NORM_SIZES(gate_norm_bwd_kernel, XT, YT, false)
        }
    }
    if (c.dw_post || c.dscale || c.dw_pre)
        column_sum_kernel<<<dim3((n + 63) / 64, 2), 1024, 0, s>>>(c, grid);
}

// F is called with the element types of (xt, yt)
template <typename C>
hipError_t by_types(const C &c, int xt, int yt, hipStream_t s, void (*f32)(const C &, hipStream_t),
                    void (*f32_h)(const C &, hipStream_t), void (*f32_b)(const C &, hipStream_t),
                    void (*h)(const C &, hipStream_t), void (*b)(const C &, hipStream_t)) {
    if (yt == SNN_F32) f32(c, s);
    else if (xt == SNN_F32) (yt == SNN_F16 ? f32_h : f32_b)(c, s);
    else (yt == SNN_F16 ? h : b)(c, s);
    return hipGetLastError();
}

template <typename T>
void run_checkpoint(int64_t rows, int n, int block, int64_t ld, void *x, int8_t *codes,
                    float *scales, bool save, hipStream_t s) {
    const int64_t per_row = ckpt_blocks(n, 128), units = rows * per_row;
    // a dimension of a launch has fewer than 2^32 threads
    const int64_t groups = (units + 15) / 16, x_groups = std::min<int64_t>(groups, 1 << 23);
    const dim3 grid((unsigned)x_groups, (unsigned)((groups + x_groups - 1) / x_groups));
    if (save)
        checkpoint_kernel<T, true><<<grid, 256, 0, s>>>(units, (uint32_t)per_row, n, block, ld,
                                                        (T *)x, codes, scales);
    else
        checkpoint_kernel<T, false><<<grid, 256, 0, s>>>(units, (uint32_t)per_row, n, block, ld,
                                                         (T *)x, codes, scales);
}

}  // namespace

size_t gate_norm_workspace_bytes(int64_t rows, int64_t n) {
    return align_up((size_t)2 * row_blocks(rows, n) * n * sizeof(float));
}

hipError_t launch_gate_norm_fwd(const GateNormFwd &c, int xt, int yt, hipStream_t s) {
    return by_types<GateNormFwd>(c, xt, yt, s, run_fwd<float, float>, run_fwd<float, half_t>,
                                 run_fwd<float, bf16_t>, run_fwd<half_t, half_t>,
                                 run_fwd<bf16_t, bf16_t>);
}

hipError_t launch_gate_norm_bwd(const GateNormBwd &c, int xt, int yt, hipStream_t s) {
    return by_types<GateNormBwd>(c, xt, yt, s, run_bwd<float, float>, run_bwd<float, half_t>,
                                 run_bwd<float, bf16_t>, run_bwd<half_t, half_t>,
                                 run_bwd<bf16_t, bf16_t>);
}

hipError_t launch_checkpoint(int64_t rows, int n, int block, int64_t ld, int dtype, void *x,
                             int8_t *codes, float *scales, bool save, hipStream_t s) {
    switch (dtype) {
        case SNN_F32: run_checkpoint<float>(rows, n, block, ld, x, codes, scales, save, s); break;
        case SNN_F16: run_checkpoint<half_t>(rows, n, block, ld, x, codes, scales, save, s); break;
        default: run_checkpoint<bf16_t>(rows, n, block, ld, x, codes, scales, save, s); break;
    }
    return hipGetLastError();
}

}  // namespace snn
