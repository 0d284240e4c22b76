// Layer norm and its backward (include/snn.h, "selective leaky block").
//
//     y = (x - mean) r w + b,  r = 1 / sqrt(mean((x - mean)^2) + eps)
//     dx = r (dy w - mean(dy w) - xhat mean(dy w xhat)) + dres,  dw = sum dy xhat
//
// Every call is one pass over HBM, which bounds it: a row stays in registers between
// its sums and the values that need them, TPR threads to a row, thread t with the NV
// runs of 8 channels 8 (i TPR + t).  The sum of squares is taken of x - mean, a second
// sum over registers: of x itself, less the mean's square, it would lose the digits
// that a mean far from zero costs.  The backward takes the statistics from x again
// (two sums more, in registers too) instead of reading stored ones.  Workgroups take
// rows in turn and hold the weights and the weights' sums of their rows; another kernel
// adds the workgroups' sums in order.  16384 rows of 2048, bf16 from and to an fp32 stream:
// forward 41 us (4.9 TB/s), backward with the stream's gradient 88 (5.3), 5 the sums.
#include "block_common.hpp"

namespace snn {
namespace {

template <int TPR>
constexpr int block_threads() { return TPR > 256 ? TPR : 256; }

// Sums over the TPR threads of a row, in a fixed order; `red` holds a slot per wave.
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

template <int TPR, int NV>
struct Row {
    int m[NV], e[NV];  // values of each run, its first channel
    __device__ inline explicit Row(int n) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            e[i] = 8 * (i * TPR + (int)threadIdx.x % TPR);
            m[i] = min(8, max(0, n - e[i]));
        }
    }
};

// x less its mean, and one over the root of its mean square, over a row of n values
// whose runs hold zeros past the end.  What the rounded mean missed is the mean of the
// differences, summed along with their squares and taken off both.
template <int TPR, int NV>
__device__ inline float centre(float (&x)[NV][8], const int (&m)[NV], float n, float eps,
                               float *red) {
    float s[1] = {0.f}, q[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += x[i][j];
    row_sum<TPR, 1>(s, red);
    const float mean = s[0] / n;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[i][j] = j < m[i] ? x[i][j] - mean : 0.f;
            q[0] += x[i][j];
            q[1] = __builtin_fmaf(x[i][j], x[i][j], q[1]);
        }
    row_sum<TPR, 2>(q, red);
    const float rest = q[0] / n;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = j < m[i] ? x[i][j] - rest : 0.f;
    return 1.f / __builtin_sqrtf(fmaxf(__builtin_fmaf(-rest, rest, q[1] / n), 0.f) + eps);
}

template <typename XT, typename YT, int TPR, int NV>
__global__ __launch_bounds__(block_threads<TPR>()) void layer_norm_kernel(LayerNorm a) {
    constexpr int RPB = block_threads<TPR>() / TPR;
    __shared__ float red[RPB][32];
    const int slot = threadIdx.x / TPR;
    const Row<TPR, NV> at(a.n);
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[i][j] = 1.f, b[i][j] = 0.f;
        if (a.w) load_run(a.w + at.e[i], at.m[i], w[i]);
        if (a.b) load_run(a.b + at.e[i], at.m[i], b[i]);
    }
    // every thread of the workgroup takes part in each round's barriers
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t row = r0 + slot;
        int m[NV];
        float x[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            m[i] = row < a.rows ? at.m[i] : 0;
            load_run(static_cast<const XT *>(a.x) + row * a.ld_x + at.e[i], m[i], x[i]);
        }
        const float r = centre<TPR, NV>(x, m, (float)a.n, a.eps, red[slot]);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = __builtin_fmaf(x[i][j] * r, w[i][j], b[i][j]);
            store_run(static_cast<YT *>(a.y) + row * a.ld_y + at.e[i], m[i], x[i]);
        }
    }
}

template <typename XT, typename YT, int TPR, int NV>
__global__ __launch_bounds__(block_threads<TPR>()) void layer_norm_bwd_kernel(LayerNormBwd q) {
    constexpr int RPB = block_threads<TPR>() / TPR;
    __shared__ float red[RPB][32];
    const LayerNorm &a = q.a;
    const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const Row<TPR, NV> at(a.n);
    const float inv_n = 1.f / (float)a.n;
    // Sums over this workgroup's rows.  Two runs of a thread have no registers for them
    // (with 1024 threads 128 a lane, 146 to 188 more in scratch): theirs are in LDS.
    constexpr bool LDS = NV > 1;
    __shared__ float held[LDS ? 2 : 1][LDS ? 8 * NV : 1][LDS ? TPR : 1];
    float w[NV][8], dw[LDS ? 1 : NV][8] = {}, db[LDS ? 1 : NV][8] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[i][j] = 1.f;
            if (LDS) held[0][8 * i + j][t] = held[1][8 * i + j][t] = 0.f;
        }
        if (a.w) load_run(a.w + at.e[i], at.m[i], w[i]);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t row = r0 + slot;
        int m[NV];
        float x[NV][8], g[NV][8];
        Raw<XT, 8> rx[NV], rr[NV];
        Raw<YT, 8> rg[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            m[i] = row < a.rows ? at.m[i] : 0;
            rx[i].load(static_cast<const XT *>(a.x) + row * a.ld_x + at.e[i], m[i]);
            rg[i].load(static_cast<const YT *>(q.gy) + row * a.ld_y + at.e[i], m[i]);
            if (q.gres)
                rr[i].load(static_cast<const XT *>(q.gres) + row * a.ld_x + at.e[i], m[i]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) rx[i].get(x[i]);
        const float r = centre<TPR, NV>(x, m, (float)a.n, a.eps, red[slot]);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            rg[i].get(g[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[i][j] *= r;
                if (LDS) {
                    held[0][8 * i + j][t] += g[i][j] * x[i][j];
                    held[1][8 * i + j][t] += g[i][j];
                } else {
                    dw[i][j] = __builtin_fmaf(g[i][j], x[i][j], dw[i][j]);
                    db[i][j] += g[i][j];
                }
                g[i][j] *= w[i][j];
                s[0] += g[i][j];
                s[1] = __builtin_fmaf(g[i][j], x[i][j], s[1]);
            }
        }
        row_sum<TPR, 2>(s, red[slot]);
        s[0] *= inv_n;
        s[1] *= inv_n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float res[8] = {};
            if (q.gres) rr[i].get(res);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                g[i][j] = __builtin_fmaf(r, g[i][j] - s[0] - x[i][j] * s[1], res[j]);
            store_run(static_cast<XT *>(q.gx) + row * a.ld_x + at.e[i], m[i], g[i]);
        }
    }
    // the workgroup's column sums, its rows' slots added in order
    __shared__ float col[RPB > 1 ? TPR * NV * 8 : 1];
    float(*sums[2])[8] = {dw, db};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float *part = q.part + ((int64_t)k * gridDim.x + blockIdx.x) * a.n;
        if constexpr (LDS) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = held[k][8 * i + j][t];
                store_run(part + at.e[i], at.m[i], v);
            }
            continue;
        }
        for (int o = 1; o < RPB; ++o) {
            __syncthreads();
            if (slot == o)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) col[j * TPR * NV + i * TPR + t] = sums[k][i][j];
            __syncthreads();
            if (slot == 0)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sums[k][i][j] += col[j * TPR * NV + i * TPR + t];
        }
        if (slot == 0)
#pragma unroll
            for (int i = 0; i < NV; ++i) store_run(part + at.e[i], at.m[i], sums[k][i]);
    }
}

// Column sums over the workgroups' partial rows, in order within each of the 16 waves'
// shares (16 loads on their way at a time), then over the waves.
__global__ __launch_bounds__(1024) void layer_norm_sum_kernel(LayerNormBwd q, int blocks) {
    float *out = blockIdx.y ? q.grad_b : q.grad_w;
    if (!out) return;  // the whole workgroup
    __shared__ float sum[16][64];
    const int n = q.a.n;
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane;
    const float *p = q.part + (int64_t)blockIdx.y * blocks * n + col;
    float s = 0.f;
    if (col < n)
        for (int b = w; b < blocks; b += 256) {
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x[i] = b + 16 * i < blocks ? p[(int64_t)(b + 16 * i) * n] : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) s += x[i];
        }
    sum[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < n) {
        for (int i = 1; i < 16; ++i) s += sum[i][lane];
        out[col] = s;
    }
}

// Threads of a row: the fewest whose runs of 8 cover it, so that a row takes one run per
// thread; two only past 8192.
int threads_per_row(int n) {
    int t = 64;
    while (t < 1024 && 8 * t < n) t *= 2;
    return t;
}

// Workgroups: as many as are resident at once, four of 256 threads to a compute unit
// (forward of 16384 rows of 2048 41 us, half as many 62); backward half as many, whose sums
// are fewer to add, where each takes eight turns at its rows or more (there and back 131 us
// against 135; 3201 rows of 1001 28 against 26) and two are left to a unit: rows past 2048
// values keep all of theirs (backward of 8192 fp32 rows of 4096 80 us, half as many 116;
// 4096 of 8192 115 and 192; 4096 of 12288 171 and 283).
int row_blocks(int64_t rows, int64_t n, bool backward) {
    const int t = threads_per_row((int)n), rpb = std::max(1, 256 / t);
    const int64_t turns = (rows + rpb - 1) / rpb;
    const int64_t most = (int64_t)4 * kPlanCus * 256 / std::max(256, t);
    const bool halve = backward && turns >= 4 * most && most / 2 >= 2 * kPlanCus;
    return (int)std::min<int64_t>(turns, halve ? most / 2 : most);
}

#define LAYER_NORM_SIZES(KERNEL, ...)                                                          \
    if (n <= 512) KERNEL<__VA_ARGS__, 64, 1><<<grid, 256, 0, s>>>(c);                          \
    else if (n <= 1024) KERNEL<__VA_ARGS__, 128, 1><<<grid, 256, 0, s>>>(c);                   \
    else if (n <= 2048) KERNEL<__VA_ARGS__, 256, 1><<<grid, 256, 0, s>>>(c);                   \
    else if (n <= 4096) KERNEL<__VA_ARGS__, 512, 1><<<grid, 512, 0, s>>>(c);                   \
    else if (n <= 8192) KERNEL<__VA_ARGS__, 1024, 1><<<grid, 1024, 0, s>>>(c);                 \
    else KERNEL<__VA_ARGS__, 1024, 2><<<grid, 1024, 0, s>>>(c);

template <typename XT, typename YT>
void run(const LayerNorm &c, hipStream_t s) {
    const int n = c.n, grid = row_blocks(c.rows, n, false);
    if (grid > 0) {
        LAYER_NORM_SIZES(layer_norm_kernel, XT, YT)
    }
}
template <typename XT, typename YT>
void run(const LayerNormBwd &c, hipStream_t s) {
    const int n = c.a.n, grid = row_blocks(c.a.rows, n, true);
    if (grid > 0) {
        LAYER_NORM_SIZES(layer_norm_bwd_kernel, XT, YT)
    }
    if (c.grad_w || c.grad_b)
        layer_norm_sum_kernel<<<dim3((n + 63) / 64, 2), 1024, 0, s>>>(c, grid);
}

template <typename C>
hipError_t by_types(const C &c, int xt, int yt, hipStream_t s) {
    if (yt == SNN_F32) run<float, float>(c, s);
    else if (xt == SNN_F32 && yt == SNN_F16) run<float, half_t>(c, s);
    else if (xt == SNN_F32) run<float, bf16_t>(c, s);
    else if (yt == SNN_F16) run<half_t, half_t>(c, s);
    else run<bf16_t, bf16_t>(c, s);
    return hipGetLastError();
}

}  // namespace

size_t layer_norm_workspace_bytes(int64_t rows, int64_t n) {
    return align_up((size_t)2 * row_blocks(rows, n, true) * n * sizeof(float));
}
hipError_t launch_layer_norm(const LayerNorm &a, int xt, int yt, hipStream_t s) {
    return by_types(a, xt, yt, s);
}
hipError_t launch_layer_norm_bwd(const LayerNormBwd &q, int xt, int yt, hipStream_t s) {
    return by_types(q, xt, yt, s);
}

}  // namespace snn
