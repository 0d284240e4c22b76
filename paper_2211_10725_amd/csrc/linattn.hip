// Linear attention with a decay per head (include/snn.h, "leaky sequence
// block"): S_t = g S_{t-1} + k_t^T v_t, o_t = scale q_t S_t.
//
// The gradients are the same recurrence with its operands exchanged (dq: q' =
// do, k' = v, v' = k, state S^T; dk: time reversed, q' = v, k' = do, v' = q,
// state R^T; dv: time reversed, q' = k, k' = q, v' = do, state R), so one
// kernel computes forward and backward; a launch runs up to kRoles of them.
#include "snn_internal.hpp"

namespace snn {
namespace {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

constexpr int kD = kLaMaxD;

template <typename T>
__device__ inline float load_value(const LaOperand &x, int t, int b, int h, int i) {
    return (float)static_cast<const T *>(
        x.p)[t * x.st + b * x.sb + (int64_t)(h / x.share) * x.sh + i];
}

// One thread per column of v, its column of the state in registers; tokens one
// after the other.
template <typename T>
__global__ __launch_bounds__(kD) void linattn_kernel(LaCall c) {
    const LaRole &r = c.role[blockIdx.z];
    const int h = blockIdx.x, b = blockIdx.y, j = threadIdx.x;
    __shared__ float qs[kD], ks[kD];
    const int len = c.lens ? min(max(c.lens[b], 0), c.T) : c.T;
    const float g = c.decay[h];
    const int64_t at = ((int64_t)b * c.H + h) * r.dk * r.dv;
    float S[kD];
#pragma unroll
    for (int i = 0; i < kD; ++i) {
        S[i] = 0.f;
        if (r.init && i < r.dk && j < r.dv)
            S[i] = r.init[at + (r.trans ? (int64_t)j * r.dk + i : (int64_t)i * r.dv + j)];
    }
    for (int n = 0; n < c.T; ++n) {
        const int t = n < len && r.reverse ? len - 1 - n : n;
        const int64_t oo = t * r.ot + b * r.ob + h * r.oh + j;
        float out = 0.f;
        if (n < len) {
            __syncthreads();
            qs[j] = j < r.dk ? load_value<T>(r.q, t, b, h, j) : 0.f;
            ks[j] = j < r.dk ? load_value<T>(r.k, t, b, h, j) : 0.f;
            __syncthreads();
            const float v = j < r.dv ? load_value<T>(r.v, t, b, h, j) * r.ws : 0.f;
#pragma unroll
            for (int i = 0; i < kD; ++i) {
                S[i] = __builtin_fmaf(ks[i], v, r.first ? S[i] * g : S[i]);
                out = __builtin_fmaf(qs[i], S[i], out);
                if (!r.first) S[i] *= g;
            }
            out *= r.rs;
        }
        if (j < r.dv) {
            if (r.o_f32) static_cast<float *>(r.o)[oo] = out;
            else static_cast<T *>(r.o)[oo] = (T)out;
        }
    }
    if (r.final_state && j < r.dv)
#pragma unroll
        for (int i = 0; i < kD; ++i)
            if (i < r.dk) r.final_state[at + (int64_t)i * r.dv + j] = S[i];
}

// dst[t,b,hk,:] = sum over the group's heads of src[t,b,h,:] (fp32, ascending)
template <typename T>
__global__ __launch_bounds__(256) void group_sum_kernel(const float *src, T *dst, int64_t st,
                                                        int64_t sb, int64_t sh, int B, int KV,
                                                        int share, int d, int64_t total) {
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (x >= total) return;
    const int d8 = d / 8;
    const int i = (int)(x % d8) * 8;
    const int64_t y = x / d8;
    const int hk = (int)(y % KV);
    const int64_t tb = y / KV;
    float s[8] = {};
    for (int m = 0; m < share; ++m) {
        const float *p = src + ((tb * KV + hk) * share + m) * d + i;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += p[e];
    }
    T *o = dst + (tb / B) * st + (tb % B) * sb + hk * sh + i;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (T)s[e];
}

// One token of every request, one workgroup each and head; thread j has column
// j of the state.
template <typename T>
__global__ __launch_bounds__(kD) void linattn_step_kernel(LaStep c) {
    const int h = blockIdx.x, b = blockIdx.y, j = threadIdx.x;
    const int slot = c.slots ? c.slots[b] : b;
    const bool idle = slot < 0 || slot >= c.n_slots;
    T *o = static_cast<T *>(c.o) + b * c.ob + h * c.oh;
    if (idle) {
        if (j < c.dv) o[j] = (T)0.f;
        return;
    }
    if (j >= c.dv) return;
    const int64_t at = ((int64_t)slot * c.H + h) * c.dk * c.dv + j;
    const float g = c.decay[h], v = load_value<T>(c.v, 0, b, h, j);
    float out = 0.f;
    for (int i = 0; i < c.dk; ++i) {
        const float k = load_value<T>(c.k, 0, b, h, i), q = load_value<T>(c.q, 0, b, h, i);
        const float s = __builtin_fmaf(k, v, c.in[at + (int64_t)i * c.dv] * g);
        c.out[at + (int64_t)i * c.dv] = s;
        out = __builtin_fmaf(q, s, out);
    }
    o[j] = (T)(out * c.scale);
}

}  // namespace

hipError_t launch_linattn(const LaCall &c, int roles, int dtype, hipStream_t s) {
    const dim3 grid(c.H, c.B, roles);
    switch (dtype) {
        case SNN_F32: linattn_kernel<float><<<grid, kD, 0, s>>>(c); break;
        case SNN_F16: linattn_kernel<half_t><<<grid, kD, 0, s>>>(c); break;
        default: linattn_kernel<bf16_t><<<grid, kD, 0, s>>>(c); break;
    }
    return hipGetLastError();
}

hipError_t launch_group_sum(const float *src, void *dst, const int64_t *stride, int T, int B,
                            int KV, int share, int d, int dtype, hipStream_t s) {
    const int64_t total = (int64_t)T * B * KV * (d / 8);
    const int grid = (int)((total + 255) / 256);
    switch (dtype) {
        case SNN_F32:
            group_sum_kernel<float><<<grid, 256, 0, s>>>(src, (float *)dst, stride[0], stride[1],
                                                         stride[2], B, KV, share, d, total);
            break;
        case SNN_F16:
            group_sum_kernel<half_t><<<grid, 256, 0, s>>>(src, (half_t *)dst, stride[0],
                                                          stride[1], stride[2], B, KV, share, d,
                                                          total);
            break;
        default:
            group_sum_kernel<bf16_t><<<grid, 256, 0, s>>>(src, (bf16_t *)dst, stride[0],
                                                          stride[1], stride[2], B, KV, share, d,
                                                          total);
    }
    return hipGetLastError();
}

hipError_t launch_linattn_step(const LaStep &c, int B, int dtype, hipStream_t s) {
    const dim3 grid(c.H, B);
    switch (dtype) {
        case SNN_F32: linattn_step_kernel<float><<<grid, kD, 0, s>>>(c); break;
        case SNN_F16: linattn_step_kernel<half_t><<<grid, kD, 0, s>>>(c); break;
        default: linattn_step_kernel<bf16_t><<<grid, kD, 0, s>>>(c); break;
    }
    return hipGetLastError();
}

}  // namespace snn
