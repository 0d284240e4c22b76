// Short causal convolution of each channel (include/snn.h, "selective leaky block").
//
//     y_t = act(bias + sum_j w_j x_{t-K+1+j})
//
// Bound by HBM: x is read and y written once.  A thread takes V neighbouring channels
// (16 bytes of a row, backward 4 channels) over a slice of tokens, with the window of the
// last K - 1 inputs in registers; four tokens' rows are on their way while four are run.
// Of a slice's rows only the K - 1 before it are read twice (by the thread of the slice
// before, at about the same time).  8 x 2048 tokens of 4096 bf16 channels, 4 taps, silu:
// forward 57 us (4.7 TB/s), backward 91 and its sums 5 (4.4; behind the forward of a
// training pass about 110).
//
// Backward in one pass over x and grad_y: the thread goes on K - 1 tokens past its
// slice, takes p = act'(.) grad_y again for each token from the window of x, and from
// the window of the last K p's the gradient of the token that left it,
//     dx_t = sum_j w_j p_{t+K-1-j},
// and adds p_t x_{t-K+1+j} to dw_j for the slice's own tokens.  The workgroup adds its
// threads' sums through LDS, another kernel those of the workgroups, both in order.
#include "block_common.hpp"

namespace snn {
namespace {

constexpr int kWaves = 4, kRuns = 64;  // a workgroup: 64 runs of channels, 4 slices
constexpr int kThreads = kWaves * kRuns;

template <typename T>
constexpr int run_of() { return 16 / (int)sizeof(T); }

struct Where {
    int b, c, m, group;  // sequence, first channel, channels, workgroup along time
    int64_t x, y;        // element offsets of (0, b, c)
};
// The last run of a row, if it is short, starts early enough to be whole, and takes some
// of its neighbour's channels along (the same values for them).  ALL: so do the threads
// past the row, where every one has to go on to a barrier.  The neighbour is one of the
// same wave where the state is updated in place: another workgroup's would write it while
// this one reads.
template <int V, bool ALL>
__device__ inline Where where(const Shortconv &a, int times) {
    Where p;
    const int cols = (a.n + kRuns * V - 1) / (kRuns * V);
    int k = blockIdx.x;
    const int col = k % cols;
    k /= cols;
    p.group = k % times;
    p.b = k / times;
    p.c = (col * kRuns + (threadIdx.x & 63)) * V;
    const int least = a.state_in && a.state_in == a.state_out ? col * kRuns * V : 0;
    if (ALL || p.c < a.n) p.c = max(least, min(p.c, a.n - V));
    p.m = min(V, max(0, a.n - p.c));
    p.x = p.b * a.x.sb + p.c;
    p.y = p.b * a.y_sb + p.c;
    return p;
}

__device__ inline int length_of(const Shortconv &a, int b) {
    return a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
}

// input i of sequence b (i >= 1 - K): from x, or before the first token from the state
template <typename T, int K, int V>
__device__ inline void input(const Shortconv &a, const Where &p, int i, float (&v)[V]) {
    if (i >= 0) {
        load_run(static_cast<const T *>(a.x.p) + p.x + i * a.x.st, p.m, v);
    } else if (a.state_in && i >= 1 - K) {
        load_run(a.state_in + ((int64_t)p.b * (K - 1) + i + K - 1) * a.n + p.c, p.m, v);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = 0.f;
    }
}

template <typename T, int V>
__device__ inline void load_whole(Raw<T, V> &r, const T *p) {
    __builtin_memcpy(r.w, p, sizeof(r.w));
}

// Groups of AHEAD tokens, the next group's rows on their way while one is run.  Those
// whose rows all lie in the sequence and whose channels all are there (`whole`) go
// without a condition: past a conditional store the compiler waits for every store before
// it when it means to wait for the loads.
template <typename T, int K>
__global__ __launch_bounds__(kThreads) void shortconv_kernel(Shortconv a, int times) {
    constexpr int V = run_of<T>(), AHEAD = 4;
    const Where p = where<V, false>(a, times);
    if (p.m <= 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = length_of(a, p.b), slice = p.group * kWaves + wave;
    const int begin = min(slice * a.slice, a.T), end = min(begin + a.slice, a.T);
    const int whole = __all(p.m == V) ? min(end, len) : begin;
    float w[K][V], bias[V] = {}, win[K][V];  // win[K - 1]: this token
#pragma unroll
    for (int j = 0; j < K; ++j) load_run(a.w + (int64_t)j * a.n + p.c, p.m, w[j]);
    if (a.bias) load_run(a.bias + p.c, p.m, bias);
    if (begin < len)
#pragma unroll
        for (int j = 1; j < K; ++j) input<T, K>(a, p, begin - K + j, win[j]);
    T *y = static_cast<T *>(a.y) + p.y;
    const T *x = static_cast<const T *>(a.x.p) + p.x;
    Raw<T, V> r[AHEAD], next[AHEAD];
    auto token = [&](const Raw<T, V> &row, float (&out)[V]) {
#pragma unroll
        for (int j = 0; j + 1 < K; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) win[j][e] = win[j + 1][e];
        row.get(win[K - 1]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            out[e] = bias[e];
#pragma unroll
            for (int j = 0; j < K; ++j) out[e] = __builtin_fmaf(w[j][e], win[j][e], out[e]);
        }
        if (a.silu)
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = silu<sizeof(T) == 4>(out[e]);
    };
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i;
            next[i].load(x + t * a.x.st, t < end && t < len ? p.m : 0);
        }
    };
    fetch(begin);
    for (int t0 = begin; t0 < end; t0 += AHEAD) {
        for (; t0 + 2 * AHEAD <= whole; t0 += AHEAD) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) r[i] = next[i];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) load_whole(next[i], x + (t0 + AHEAD + i) * a.x.st);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                float out[V];
                token(r[i], out);
                store_run(y + (t0 + i) * a.y_st, V, out);
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) r[i] = next[i];
        if (t0 + AHEAD < end) fetch(t0 + AHEAD);
        if (t0 + AHEAD <= whole) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                float out[V];
                token(r[i], out);
                store_run(y + (t0 + i) * a.y_st, V, out);
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (t0 + i >= end) break;
            float out[V];
            token(r[i], out);
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = t0 + i < len ? out[e] : 0.f;
            store_run(y + (t0 + i) * a.y_st, p.m, out);
        }
    }
    // the last inputs, by the thread that also reads the state (which may be the same)
    if (a.state_out && slice == 0) {
        float v[K - 1][V];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) input<T, K>(a, p, len - K + 1 + j, v[j]);
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
            store_run(a.state_out + ((int64_t)p.b * (K - 1) + j) * a.n + p.c, p.m, v[j]);
    }
}

template <typename T, int K, int V>
__global__ __launch_bounds__(kThreads) void shortconv_bwd_kernel(ShortconvBwd q, int times) {
    constexpr int AHEAD = 4;
    const Shortconv &a = q.a;
    const Where p = where<V, true>(a, times);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = length_of(a, p.b), slice = p.group * kWaves + wave;
    const int begin = min(slice * a.slice, a.T), end = min(begin + a.slice, a.T);
    // the first slice goes on to the gradients of the state's rows
    const int stop = begin < end || slice == 0 ? end + K - 1 : begin;
    const int whole = __all(p.m == V) ? min(end, len) : begin;
    float w[K][V], bias[V] = {}, win[K][V] = {}, ps[K][V] = {}, dw[K][V] = {}, db[V] = {};
#pragma unroll
    for (int j = 0; j < K; ++j) load_run(a.w + (int64_t)j * a.n + p.c, p.m, w[j]);
    if (a.bias) load_run(a.bias + p.c, p.m, bias);
    if (begin < len)
#pragma unroll
        for (int j = 1; j < K; ++j) input<T, K>(a, p, begin - K + j, win[j]);
    const T *x = static_cast<const T *>(a.x.p) + p.x, *gy = static_cast<const T *>(q.gy) + p.y;
    T *gx = static_cast<T *>(q.gx) + p.x;
    Raw<T, V> rx[AHEAD], rg[AHEAD], nx[AHEAD], ng[AHEAD];
    // the window a token on: its p, where it lies in the sequence
    auto token = [&](const Raw<T, V> &xrow, const Raw<T, V> &grow, bool in) {
        float g[V];
#pragma unroll
        for (int j = 0; j + 1 < K; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) win[j][e] = win[j + 1][e], ps[j][e] = ps[j + 1][e];
        xrow.get(win[K - 1]);
        grow.get(g);
        if (a.silu)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float s = bias[e], act, slope;
#pragma unroll
                for (int j = 0; j < K; ++j) s = __builtin_fmaf(w[j][e], win[j][e], s);
                silu_slope<sizeof(T) == 4>(s, act, slope);
                g[e] *= slope;
            }
#pragma unroll
        for (int e = 0; e < V; ++e) ps[K - 1][e] = in ? g[e] : 0.f;
    };
    auto add_sums = [&]() {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            db[e] += ps[K - 1][e];
#pragma unroll
            for (int j = 0; j < K; ++j)
                dw[j][e] = __builtin_fmaf(ps[K - 1][e], win[j][e], dw[j][e]);
        }
    };
    auto input_grad = [&](float (&out)[V]) {  // of the input that left the window
#pragma unroll
        for (int e = 0; e < V; ++e) {
            out[e] = 0.f;
#pragma unroll
            for (int j = 0; j < K; ++j) out[e] = __builtin_fmaf(w[j][e], ps[K - 1 - j][e], out[e]);
        }
    };
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i, k = t < stop && t < len ? p.m : 0;
            nx[i].load(x + t * a.x.st, k);
            ng[i].load(gy + t * a.y_st, k);
        }
    };
    fetch(begin);
    for (int t0 = begin; t0 < stop; t0 += AHEAD) {
        // whole groups, past the tokens whose window began in another slice (shortconv_kernel)
        for (; t0 >= begin + K - 1 && t0 + 2 * AHEAD <= whole; t0 += AHEAD) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) rx[i] = nx[i], rg[i] = ng[i];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                load_whole(nx[i], x + (t0 + AHEAD + i) * a.x.st);
                load_whole(ng[i], gy + (t0 + AHEAD + i) * a.y_st);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                float out[V];
                token(rx[i], rg[i], true);
                add_sums();
                input_grad(out);
                store_run(gx + (t0 + i - K + 1) * a.x.st, V, out);
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) rx[i] = nx[i], rg[i] = ng[i];
        if (t0 + AHEAD < stop) fetch(t0 + AHEAD);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i;
            if (t >= stop) break;
            token(rx[i], rg[i], t < len);
            if (t < end && t < len) add_sums();
            const int from = t - K + 1;  // the input that left the window
            if (from < begin && slice > 0) continue;
            float out[V];
            input_grad(out);
            const int row = from - (len - K + 1);  // of the state after the sequence
            if (q.grad_state_out && row >= 0 && row < K - 1) {
                float v[V];
                load_run(q.grad_state_out + ((int64_t)p.b * (K - 1) + row) * a.n + p.c, p.m, v);
#pragma unroll
                for (int e = 0; e < V; ++e) out[e] += v[e];
            }
            if (from >= 0) {
                if (from >= len)
#pragma unroll
                    for (int e = 0; e < V; ++e) out[e] = 0.f;
                store_run(gx + from * a.x.st, p.m, out);
            } else if (q.grad_state_in) {
                store_run(q.grad_state_in + ((int64_t)p.b * (K - 1) + from + K - 1) * a.n + p.c,
                          p.m, out);
            }
        }
    }
    if (!q.grad_w && !q.grad_bias) return;
    __shared__ float sum[kWaves][V][kRuns];
    const int lane = threadIdx.x & 63;
    float *part = q.part + (int64_t)(p.b * times + p.group) * (K + 1) * a.n + p.c;
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) sum[wave][e][lane] = j < K ? dw[j < K ? j : 0][e] : db[e];
        __syncthreads();
        if (wave == 0) {
            float s[V];
#pragma unroll
            for (int e = 0; e < V; ++e)
                s[e] = sum[0][e][lane] + sum[1][e][lane] + sum[2][e][lane] + sum[3][e][lane];
            store_run(part + (int64_t)j * a.n, p.m, s);
        }
    }
}

// Gradients of w and bias: the workgroups' sums, in order within each of the 16 waves'
// shares, then over the waves.
__global__ __launch_bounds__(1024) void shortconv_sum_kernel(ShortconvBwd q, int width, int rows) {
    __shared__ float sum[16][64];
    const int64_t size = (int64_t)(width + 1) * q.a.n;
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t e = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.f;
    if (e < size)
        for (int r = w; r < rows; r += 128) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = r + 16 * i < rows ? q.part[(r + 16 * i) * size + e] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[i];
        }
    sum[w][lane] = s;
    __syncthreads();
    if (w == 0 && e < size) {
        for (int i = 1; i < 16; ++i) s += sum[i][lane];
        const int64_t taps = (int64_t)width * q.a.n;
        if (e < taps && q.grad_w) q.grad_w[e] = s;
        if (e >= taps && q.grad_bias) q.grad_bias[e - taps] = s;
    }
}

// One token: a thread takes V channels of a request.
template <typename T, int K>
__global__ __launch_bounds__(256) void shortconv_step_kernel(Shortconv a, const int32_t *slots,
                                                             int n_slots) {
    constexpr int V = 4;
    const int per = (a.n + 256 * V - 1) / (256 * V), b = blockIdx.x / per;
    const int c = ((blockIdx.x - b * per) * 256 + threadIdx.x) * V, m = min(V, a.n - c);
    if (m <= 0) return;
    T *y = static_cast<T *>(a.y) + b * a.y_sb + c;
    const int slot = slots ? slots[b] : b;
    float out[V] = {};
    if (slot >= 0 && slot < n_slots) {
        const int64_t at = (int64_t)slot * (K - 1) * a.n + c;
        float v[K][V], w[K][V];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) load_run(a.state_in + at + (int64_t)j * a.n, m, v[j]);
        load_run(static_cast<const T *>(a.x.p) + b * a.x.sb + c, m, v[K - 1]);
#pragma unroll
        for (int j = 0; j < K; ++j) load_run(a.w + (int64_t)j * a.n + c, m, w[j]);
        if (a.bias) load_run(a.bias + c, m, out);
#pragma unroll
        for (int e = 0; e < V; ++e) {
#pragma unroll
            for (int j = 0; j < K; ++j) out[e] = __builtin_fmaf(w[j][e], v[j][e], out[e]);
            if (a.silu) out[e] = silu<sizeof(T) == 4>(out[e]);
        }
#pragma unroll
        for (int j = 0; j < K - 1; ++j) store_run(a.state_out + at + (int64_t)j * a.n, m, v[j + 1]);
    }
    store_run(y, m, out);
}

// Tokens of a thread: `most`, fewer (not below the window) while that leaves the device
// with less than eight waves to a compute unit.  8 x 2048 tokens of 4096 bf16 channels:
// forward in slices of 64 57 us (32: 64), backward with its sums, whose threads go on past
// their slice, of 128 95 us (64: 102, 32: 102).
constexpr int kMostFwd = 64, kMostBwd = 128;
struct Plan {
    int slice, times, cols;
};
Plan plan_of(int T, int B, int n, int runs, int most) {
    Plan p;
    p.cols = (n + kRuns * runs - 1) / (kRuns * runs);
    p.slice = most;
    while (p.slice > 8 &&
           (int64_t)p.cols * B * ((T + kWaves * p.slice - 1) / (kWaves * p.slice)) < 2 * kPlanCus)
        p.slice /= 2;
    p.times = std::max(1, (T + kWaves * p.slice - 1) / (kWaves * p.slice));
    return p;
}

template <typename T, int K>
void run_fwd(const Shortconv &a, hipStream_t s) {
    const Plan p = plan_of(a.T, a.B, a.n, run_of<T>(), kMostFwd);
    Shortconv c = a;
    c.slice = p.slice;
    shortconv_kernel<T, K><<<(unsigned)(p.cols * p.times * a.B), kThreads, 0, s>>>(c, p.times);
}
template <typename T, int K>
void run_bwd(const ShortconvBwd &q, hipStream_t s) {
    const Plan p = plan_of(q.a.T, q.a.B, q.a.n, 4, kMostBwd);
    ShortconvBwd c = q;
    c.a.slice = p.slice;
    if (q.a.B > 0)
        shortconv_bwd_kernel<T, K, 4>
            <<<(unsigned)(p.cols * p.times * q.a.B), kThreads, 0, s>>>(c, p.times);
    if (q.grad_w || q.grad_bias)
        shortconv_sum_kernel<<<(unsigned)(((int64_t)(K + 1) * q.a.n + 63) / 64), 1024, 0, s>>>(
            c, K, p.times * q.a.B);
}
template <typename T, int K>
void run_step(const Shortconv &a, const int32_t *slots, int n_slots, hipStream_t s) {
    shortconv_step_kernel<T, K><<<a.B * ((a.n + 1023) / 1024), 256, 0, s>>>(a, slots, n_slots);
}

#define SHORTCONV_WIDTHS(RUN, T, ...)           \
    switch (width) {                            \
        case 2: RUN<T, 2>(__VA_ARGS__); break;  \
        case 3: RUN<T, 3>(__VA_ARGS__); break;  \
        case 4: RUN<T, 4>(__VA_ARGS__); break;  \
        case 5: RUN<T, 5>(__VA_ARGS__); break;  \
        case 6: RUN<T, 6>(__VA_ARGS__); break;  \
        case 7: RUN<T, 7>(__VA_ARGS__); break;  \
        default: RUN<T, 8>(__VA_ARGS__); break; \
    }
#define SHORTCONV_TYPES(RUN, ...)                                       \
    switch (dtype) {                                                    \
        case SNN_F32: SHORTCONV_WIDTHS(RUN, float, __VA_ARGS__) break;  \
        case SNN_F16: SHORTCONV_WIDTHS(RUN, half_t, __VA_ARGS__) break; \
        default: SHORTCONV_WIDTHS(RUN, bf16_t, __VA_ARGS__) break;      \
    }

}  // namespace

size_t shortconv_workspace_bytes(int T, int B, int n, int width) {
    const Plan p = plan_of(T, B, n, 4, kMostBwd);
    return align_up((size_t)p.times * B * (width + 1) * n * sizeof(float));
}

hipError_t launch_shortconv(const Shortconv &a, int width, int dtype, hipStream_t s) {
    SHORTCONV_TYPES(run_fwd, a, s)
    return hipGetLastError();
}
hipError_t launch_shortconv_bwd(const ShortconvBwd &q, int width, int dtype, hipStream_t s) {
    SHORTCONV_TYPES(run_bwd, q, s)
    return hipGetLastError();
}
hipError_t launch_shortconv_step(const Shortconv &a, const int32_t *slots, int n_slots, int width,
                                 int dtype, hipStream_t s) {
    SHORTCONV_TYPES(run_step, a, slots, n_slots, s)
    return hipGetLastError();
}

}  // namespace snn
