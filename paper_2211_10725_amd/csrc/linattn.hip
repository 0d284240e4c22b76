// Linear attention with a decay per head (include/snn.h, "leaky sequence
// block"): S_t = g S_{t-1} + k_t^T v_t, o_t = scale q_t S_t.
//
// The gradients are the same recurrence with its operands exchanged (dq: q' =
// do, k' = v, v' = k, state S^T; dk: time reversed, q' = v, k' = do, v' = q,
// state R^T; dv: time reversed, q' = k, k' = q, v' = do, state R), so one
// kernel computes forward and backward; a launch runs up to kLaRoles of them.
//
// Whole sequences go in chunks of C tokens (64 of 16 bits, 32 of fp32) with the
// state between them, all of it on the matrix cores:
//   o_i = rs (sum_{j<=i} g^{i-j} ws (q_i.k_j) v_j + g^{i+first} q_i X)
//   X'  = g^C X + sum_j g^{C-first-j} ws k_j^T v_j
// A wave owns 32 columns of v and the state's columns with them, in registers,
// so waves exchange nothing but the staged tiles of q, k and v; each computes
// the chunk's scores q.k for itself (18 % of its products at d = 128).  Every
// product is arranged so that a result lies in the registers as the next
// product's operand: scores and output are taken transposed (s x t, dv x t), and
// the 16 rows of a result tile are the k values 4 g + r that lane group g holds
// of an operand, in whatever order, as long as both operands agree on it.
//
// 16-bit operands multiply exactly into fp32.  What is fp32 and becomes an
// operand is split: scores and state into two 16-bit parts (2^-16 of a term,
// far under the result's own rounding), v g^j in the state's update into as many
// as keep fp32's precision (three bf16, two fp16).  fp16 parts are taken after a
// scaling by a power of two that puts the wave's largest value near 2^14, so
// neither large sums nor small ones leave the type's range.
//
// A masked score is replaced by zero, but a zero times a later token's infinite
// or NaN value would still reach earlier outputs: where a chunk's v holds
// one, its tokens go one at a time.
//
// Few heads: the tokens are cut into segments, a first launch takes every
// segment's own state, a second adds them up (decayed), a third computes the
// outputs from each segment's state.
#include <type_traits>

#include "snn_internal.hpp"

namespace snn {
namespace {

typedef _Float16 half_t;
typedef __bf16 bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// decay^e, e >= 0, by repeated squaring in fp64 (0^0 = 1)
__device__ inline float decay_power(float g, int e) {
    double r = 1.0, b = g;
    for (; e; e >>= 1, b *= b)
        if (e & 1) r *= b;
    return (float)r;
}

__device__ inline float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// largest of 64 lanes' values >= 0, the same in every lane
__device__ inline float wave_max(float x) {
#define SNN_DPP_MAX(ctrl)                                                                         \
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, \
                                                            false)))
    SNN_DPP_MAX(0x111);  // row_shr:1, 2, 4, 8: lane 15 of each row has the row's
    SNN_DPP_MAX(0x112);
    SNN_DPP_MAX(0x114);
    SNN_DPP_MAX(0x118);
    SNN_DPP_MAX(0x142);  // row_bcast:15, 31: lane 63 has them all
    SNN_DPP_MAX(0x143);
#undef SNN_DPP_MAX
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// The exponent e for which x 2^e lies in [2^14, 2^15), within [-120, 120]
__device__ inline int scale_to_half(float x) {
    return min(120, max(-120, 14 + 127 - (int)((__float_as_uint(x) >> 23) & 255u)));
}

template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8)));
};

template <typename T>
__device__ inline f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    typedef typename Vec8<T>::type v;
    if constexpr (std::is_same_v<T, half_t>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v, a),
                                                      __builtin_bit_cast(v, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v, a),
                                                       __builtin_bit_cast(v, b), c, 0, 0, 0);
}
__device__ inline f32x4 mfma(float a, float b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <typename T>
__device__ inline u32x4 pack(const float (&x)[8]) {
    typename Vec8<T>::type v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (T)x[j];
    return __builtin_bit_cast(u32x4, v);
}
// the next part of x: its nearest 16-bit values, taken off x
template <typename T>
__device__ inline u32x4 take_part(float (&x)[8]) {
    const u32x4 p = pack<T>(x);
    const auto v = __builtin_bit_cast(typename Vec8<T>::type, p);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] -= (float)v[j];
    return p;
}
template <typename T>
__device__ inline void unpack(const u32x4 &p, float (&x)[8]) {
    const auto v = __builtin_bit_cast(typename Vec8<T>::type, p);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
}

// ---- geometry ----------------------------------------------------------------------
// D: head sizes up to 64 or 128, padded with zeros.  A wave has 32 columns, so
// D / 32 waves make a workgroup; each thread stages four 16-byte runs of every
// tile.
template <typename T, int D>
struct Geo {
    static constexpr bool kHalf = sizeof(T) == 2;
    static constexpr int C = kHalf ? 64 : 32;         // tokens of a chunk
    static constexpr int kWaves = D / 32, kThreads = 64 * kWaves;
    static constexpr int kRun = 16 / sizeof(T);       // values of a 16-byte run
    static constexpr int kRuns = D / kRun;            // runs of a row
    static constexpr int kRows = kThreads / kRuns;    // rows that the threads stage at once
    static constexpr int kVec = C / kRows;            // runs a thread stages
    static_assert(kVec == 4);
    // 16-bit rows: run c of row r lies at slot c ^ swz(r), so that the 16 rows that
    // a fragment's lanes read at one run, and the 4 rows by 4 runs of a transposing
    // read, fall on distinct banks.  fp32 rows: 4 values of padding, which spread
    // both the 16 rows of a 16-byte read and the 4 rows of a 4-byte read.
    static constexpr int kStride = kHalf ? D : D + 4;
    static constexpr int kTile = C * kStride;
    __device__ static inline int swz(int r) {
        if constexpr (!kHalf) return 0;
        else if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
        else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    }
    __device__ static inline int at(int r, int run) {
        return r * kStride + (run ^ swz(r)) * kRun;
    }
};

// Rows of one operand for this workgroup's sequence and head: token n of the
// recurrence lies at base + n step.
template <typename T, int D>
struct Source {
    const T *lane;  // run and first row of this thread
    int64_t step;
    bool live;      // this thread's run lies within the head
    __device__ inline void init(const LaOperand &x, int b, int h, int width, int last) {
        typedef Geo<T, D> G;
        const int run = threadIdx.x % G::kRuns, row = threadIdx.x / G::kRuns;
        step = last >= 0 ? -x.st : x.st;
        lane = static_cast<const T *>(x.p) + b * x.sb + (int64_t)(h / x.share) * x.sh +
               (last >= 0 ? last * x.st : 0) + row * step + run * G::kRun;
        live = run * G::kRun < width;
    }
    __device__ inline void load(int n, int count, u32x4 (&v)[4]) const {
        typedef Geo<T, D> G;
        const int row = threadIdx.x / G::kRuns;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = u32x4{0, 0, 0, 0};
            if (live && row + i * G::kRows < count)
                v[i] = *reinterpret_cast<const u32x4 *>(lane + (int64_t)(n + i * G::kRows) * step);
        }
    }
    __device__ static inline void stage(T *tile, const u32x4 (&v)[4]) {
        typedef Geo<T, D> G;
        const int run = threadIdx.x % G::kRuns, row = threadIdx.x / G::kRuns;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x4 *>(tile + G::at(row + i * G::kRows, run)) = v[i];
    }
};

// whether a staged run holds an infinity or NaN
template <typename T>
__device__ inline bool not_finite(const u32x4 (&v)[4]) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (std::is_same_v<T, float>)
                bad |= (v[i][j] & 0x7f800000u) + 0x00800000u;
            else if constexpr (std::is_same_v<T, half_t>)
                bad |= (v[i][j] & 0x7c007c00u) + 0x04000400u;
            else
                bad |= (v[i][j] & 0x7f807f80u) + 0x00800080u;
        }
    return (bad & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u)) != 0;
}

// 8 values of column `col` (of 16 lanes' columns each) in rows 32 u + 4 g .. + 3
// and 32 u + 16 + 4 g .. + 3 of a row-major tile: within 16 lanes, the
// transposing read hands lane i element e of lane 4 e + i / 4's 4-value run
// (position i % 4), so lane L points at row 4 g + L / 4 and the run of lanes
// 4 (L % 4) .. + 3.  Pair p of 16 columns holds columns 8 (i / 4) + 4 p + i % 4
// of 32: a lane's results of both pairs are 8 neighbours in memory.
template <typename T, int D>
__device__ inline u32x4 read_columns(const T *tile, int u, int block, int p) {
    typedef Geo<T, D> G;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int lane = threadIdx.x & 63, g = lane >> 4, L = lane & 15;
    const int row = 32 * u + 4 * g + (L >> 2);
    const T *a = tile + G::at(row, 4 * block + (L & 3)) + 4 * p;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(a + 16 * G::kStride));
    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
    return u32x4{x[0], x[1], y[0], y[1]};
}

// The state's columns of one wave: tile (a, p) holds rows row(a) + r and column
// col(p), r = 0 .. 3.
template <typename T, int D>
struct State {
    static constexpr int kTiles = D / 16;
    f32x4 s[kTiles][2];
    __device__ static inline int row(int a) {
        const int g = (threadIdx.x & 63) >> 4;
        return sizeof(T) == 2 ? 32 * (a >> 1) + 8 * g + 4 * (a & 1) : 16 * a + 4 * g;
    }
    __device__ static inline int col(int p) {
        const int w = threadIdx.x >> 6, i = threadIdx.x & 15;
        return 32 * w + (sizeof(T) == 2 ? 8 * (i >> 2) + 4 * p + (i & 3) : 16 * p + i);
    }
    __device__ inline void load(const float *from, bool trans, int dk, int dv) {
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                s[a][p] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (!from || row(a) >= dk || col(p) >= dv) continue;
                if (trans) {
                    s[a][p] = *reinterpret_cast<const f32x4 *>(from + (int64_t)col(p) * dk + row(a));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[a][p][r] = from[(int64_t)(row(a) + r) * dv + col(p)];
                }
            }
    }
    __device__ inline void store(float *to, int dk, int dv) const {
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (row(a) < dk && col(p) < dv)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        to[(int64_t)(row(a) + r) * dv + col(p)] = s[a][p][r];
    }
    __device__ inline void scale(float f) {
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < 2; ++p) s[a][p] *= f;
    }
    // largest finite magnitude of the wave's part
    __device__ inline float largest() const {
        float m = 0.f;
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = fmaxf(m, __builtin_fabsf(s[a][p][r]));
        m = wave_max(m);
        if (m < __builtin_inff()) return m;
        m = 0.f;
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = __builtin_fabsf(s[a][p][r]);
                    if (x < __builtin_inff()) m = fmaxf(m, x);
                }
        return wave_max(m);
    }
};

// One workgroup: one role, sequence, head and segment.  OUT: outputs (and the
// final state); else the segment's own state alone, into its slot.
template <typename T, int D, bool OUT>
__global__ __launch_bounds__(2 * D, 2) void linattn_kernel(LaCall c) {
    typedef Geo<T, D> G;
    constexpr int C = G::C, kTT = C / 16;  // tiles of 16 tokens
    constexpr bool kHalf = G::kHalf, kNorm = std::is_same_v<T, half_t>;
    __shared__ __attribute__((aligned(16))) T tq[OUT ? G::kTile : 8], tk[G::kTile], tv[G::kTile];
    __shared__ float pw[C + 1];       // decay^i
    __shared__ float weight[2 * C];   // ws decay^(C - first - x), zero from x = C on
    __shared__ int flag[2];

    const int item = xcd_local_item();
    const LaRole &r = c.role[item % c.roles];
    const int seg = item / c.roles % c.segs, bh = item / c.roles / c.segs;
    const int b = bh / c.H, h = bh % c.H;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 15, g = lane >> 4;
    const int len = c.lens ? min(max(c.lens[b], 0), c.T) : c.T;
    const int begin = seg * c.seg_len, end = (int)min((int64_t)begin + c.seg_len, (int64_t)len);
    const int dk = r.dk, dv = r.dv;
    const float decay = c.decay[h];
    for (int i = tid; i <= C; i += G::kThreads) pw[i] = decay_power(decay, i);
    for (int i = tid; i < 2 * C; i += G::kThreads)
        weight[i] = i < C ? r.ws * decay_power(decay, max(C - r.first - i, 0)) : 0.f;
    if (tid < 2) flag[tid] = 0;

    Source<T, D> sq, sk, sv;
    const int last = r.reverse ? len - 1 : -1;  // len 0: no token is read
    if (OUT) sq.init(r.q, b, h, dk, last);
    sk.init(r.k, b, h, dk, last);
    sv.init(r.v, b, h, dv, last);

    State<T, D> S;
    const int64_t at = (int64_t)bh * dk * dv;
    S.load(OUT && r.init ? r.init + seg * r.init_seg + at : nullptr, r.trans, dk, dv);
    int exp_s = 0;  // fp16: the state is s 2^-exp_s

    u32x4 q4[4], k4[4], v4[4];
    if (OUT) sq.load(begin, end - begin, q4);
    sk.load(begin, end - begin, k4);
    sv.load(begin, end - begin, v4);
    int par = 0;
    for (int n = begin; n < end; par ^= 1) {
        int count = min(C, end - n);
        __syncthreads();  // the previous chunk's reads are done
        if (OUT) Source<T, D>::stage(tq, q4);
        Source<T, D>::stage(tk, k4);
        Source<T, D>::stage(tv, v4);
        if (OUT && __any(not_finite<T>(v4)) && lane == 0) flag[par] = 1;
        __syncthreads();
        if (OUT && flag[par]) {  // the whole workgroup: one token alone
            count = 1;
            for (int i = tid; i < G::kTile; i += G::kThreads)
                if (i >= G::kStride) tk[i] = (T)0.f, tv[i] = (T)0.f;
            __syncthreads();
        }
        if (tid == 0) flag[par ^ 1] = 0;
        const int next = n + count, left = end - next;
        const float gc = pw[count];
        float largest = 0.f;
        if constexpr (kNorm) largest = S.largest();

        if constexpr (kHalf) {
            u32x4 vf[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int p = 0; p < 2; ++p) vf[u][p] = read_columns<T, D>(tv, u, wave, p);
            if constexpr (OUT) {
                f32x4 O[kTT][2], P[kTT][kTT];
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
#pragma unroll
                    for (int p = 0; p < 2; ++p) O[t][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s <= t; ++s) P[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                int exp_x = 0;
                if constexpr (kNorm) exp_x = scale_to_half(largest);
                const float fx = pow2(exp_x);
#pragma unroll
                for (int q = 0; q < D / 32; ++q) {
                    u32x4 qf[kTT], kf[kTT];
#pragma unroll
                    for (int t = 0; t < kTT; ++t) {
                        const int x = G::at(16 * t + l, 4 * q + g);
                        qf[t] = *reinterpret_cast<const u32x4 *>(tq + x);
                        kf[t] = *reinterpret_cast<const u32x4 *>(tk + x);
                    }
#pragma unroll
                    for (int t = 0; t < kTT; ++t)
#pragma unroll
                        for (int s = 0; s <= t; ++s) P[t][s] = mfma<T>(kf[s], qf[t], P[t][s]);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        float x[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            x[j] = S.s[2 * q + (j >> 2)][p][j & 3];
                            if constexpr (kNorm) x[j] *= fx;
                        }
                        const u32x4 hi = take_part<T>(x), lo = pack<T>(x);
#pragma unroll
                        for (int t = 0; t < kTT; ++t) {
                            O[t][p] = mfma<T>(lo, qf[t], O[t][p]);
                            O[t][p] = mfma<T>(hi, qf[t], O[t][p]);
                        }
                    }
                }
                sq.load(next, left, q4);  // the next chunk, on its way meanwhile
                sk.load(next, left, k4);
                sv.load(next, left, v4);
                // scores: decayed, those of later tokens zero
                const float ps = r.rs * r.ws;
                float near[4], far[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int d = l - 4 * g - x;
                    near[x] = ps * pw[max(d, 0)];
                    far[x] = ps * pw[16 + d];
                }
                float most = 0.f;
#pragma unroll
                for (int t = 0; t < kTT; ++t)
#pragma unroll
                    for (int s = 0; s <= t; ++s)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            float e = P[t][s][x];
                            if (s == t) e = l - 4 * g - x >= 0 ? e * near[x] : 0.f;
                            else if (s + 1 == t) e *= far[x];
                            else e *= far[x] * pw[16 * (t - s - 1)];
                            P[t][s][x] = e;
                            if constexpr (kNorm) {
                                const float a = __builtin_fabsf(e);
                                most = fmaxf(most, a < __builtin_inff() ? a : 0.f);
                            }
                        }
                int exp_p = 0;
                // at most 60: what smaller scores lose is far below an fp16 output's least step
                if constexpr (kNorm) exp_p = min(60, scale_to_half(wave_max(most)));
                const float fp = pow2(exp_p), back = pow2(-exp_p);
                const float row = r.rs * pw[l] * (r.first ? decay : 1.f);
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
                    float f = row * pw[16 * t];
                    if constexpr (kNorm) f = __builtin_ldexpf(f, exp_p - exp_x - exp_s);
#pragma unroll
                    for (int p = 0; p < 2; ++p) O[t][p] *= f;
#pragma unroll
                    for (int u = 0; u <= t / 2; ++u) {
                        float x[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int s = 2 * u + (j >> 2);
                            x[j] = s <= t ? P[t][s <= t ? s : 0][j & 3] : 0.f;
                            if constexpr (kNorm) x[j] *= fp;
                        }
                        const u32x4 hi = take_part<T>(x), lo = pack<T>(x);
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            O[t][p] = mfma<T>(vf[u][p], lo, O[t][p]);
                            O[t][p] = mfma<T>(vf[u][p], hi, O[t][p]);
                        }
                    }
                    // token 16 t + l, columns 8 g .. 8 g + 7 of the wave's 32
                    const int tok = 16 * t + l, col = 32 * wave + 8 * g;
                    if (tok < count && col < dv) {
                        const int64_t to = (r.reverse ? len - 1 - (n + tok) : n + tok) * r.ot +
                                           b * r.ob + h * r.oh + col;
                        if constexpr (kNorm) O[t][0] *= back, O[t][1] *= back;
                        if (r.o_f32) {
                            f32x4 *o = reinterpret_cast<f32x4 *>(static_cast<float *>(r.o) + to);
                            o[0] = O[t][0];
                            o[1] = O[t][1];
                        } else {
                            const float x[8] = {O[t][0][0], O[t][0][1], O[t][0][2], O[t][0][3],
                                                O[t][1][0], O[t][1][1], O[t][1][2], O[t][1][3]};
                            *reinterpret_cast<u32x4 *>(static_cast<T *>(r.o) + to) = pack<T>(x);
                        }
                    }
                }
            } else {
                sk.load(next, left, k4);
                sv.load(next, left, v4);
            }
            // the state's update
            float w[2][2][8], most = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    unpack<T>(vf[u][p], w[u][p]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        w[u][p][j] *= weight[32 * u + 16 * (j >> 2) + 4 * g + (j & 3) + C - count];
                        if constexpr (kNorm) {
                            const float a = __builtin_fabsf(w[u][p][j]);
                            most = fmaxf(most, a < __builtin_inff() ? a : 0.f);
                        }
                    }
                }
            if constexpr (kNorm) {
                // the scale of this chunk's v g^j, unless the state would leave 2^61
                most = wave_max(most);
                int e = most > 0.f ? scale_to_half(most) : exp_s;
                const float left_s = largest * __builtin_fabsf(gc);
                if (left_s > 0.f)
                    e = min(e, exp_s + min(120, scale_to_half(left_s) + 46));
                S.scale(left_s > 0.f ? __builtin_ldexpf(gc, e - exp_s) : 0.f);
                exp_s = e;
            } else {
                S.scale(gc);
            }
            constexpr int kParts = kNorm ? 2 : 3;
            const float fv = pow2(exp_s);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 part[2][kParts];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    if constexpr (kNorm)
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[u][p][j] *= fv;
#pragma unroll
                    for (int m = 0; m < kParts; ++m) part[p][m] = take_part<T>(w[u][p]);
                }
#pragma unroll
                for (int a = 0; a < State<T, D>::kTiles; ++a) {
                    const u32x4 kt = read_columns<T, D>(tk, u, a >> 1, a & 1);
#pragma unroll
                    for (int m = kParts - 1; m >= 0; --m)
#pragma unroll
                        for (int p = 0; p < 2; ++p) S.s[a][p] = mfma<T>(kt, part[p][m], S.s[a][p]);
                }
            }
        } else {
            const float *fq = reinterpret_cast<const float *>(tq),
                        *fk = reinterpret_cast<const float *>(tk),
                        *fv = reinterpret_cast<const float *>(tv);
            f32x4 vf[kTT][2];
#pragma unroll
            for (int s = 0; s < kTT; ++s)
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        vf[s][p][x] = fv[(16 * s + 4 * g + x) * G::kStride + 32 * wave + 16 * p + l];
            if constexpr (OUT) {
                f32x4 O[kTT][2], P[kTT][kTT];
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
#pragma unroll
                    for (int p = 0; p < 2; ++p) O[t][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s <= t; ++s) P[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int a = 0; a < State<T, D>::kTiles; ++a) {
                    f32x4 qf[kTT], kf[kTT];
#pragma unroll
                    for (int t = 0; t < kTT; ++t) {
                        const int x = (16 * t + l) * G::kStride + 16 * a + 4 * g;
                        qf[t] = *reinterpret_cast<const f32x4 *>(fq + x);
                        kf[t] = *reinterpret_cast<const f32x4 *>(fk + x);
                    }
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int t = 0; t < kTT; ++t) {
#pragma unroll
                            for (int s = 0; s <= t; ++s)
                                P[t][s] = mfma(kf[s][x], qf[t][x], P[t][s]);
#pragma unroll
                            for (int p = 0; p < 2; ++p)
                                O[t][p] = mfma(S.s[a][p][x], qf[t][x], O[t][p]);
                        }
                }
                sq.load(next, left, q4);
                sk.load(next, left, k4);
                sv.load(next, left, v4);
                const float ps = r.rs * r.ws, row = r.rs * pw[l] * (r.first ? decay : 1.f);
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
#pragma unroll
                    for (int p = 0; p < 2; ++p) O[t][p] *= row * pw[16 * t];
#pragma unroll
                    for (int s = 0; s <= t; ++s)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int d = 16 * (t - s) + l - 4 * g - x;
                            const float e = d >= 0 ? P[t][s][x] * (ps * pw[max(d, 0)]) : 0.f;
#pragma unroll
                            for (int p = 0; p < 2; ++p) O[t][p] = mfma(vf[s][p][x], e, O[t][p]);
                        }
                    const int tok = 16 * t + l;
                    if (tok < count)
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const int col = 32 * wave + 16 * p + 4 * g;
                            if (col < dv)
                                *reinterpret_cast<f32x4 *>(
                                    static_cast<float *>(r.o) +
                                    (r.reverse ? len - 1 - (n + tok) : n + tok) * r.ot + b * r.ob +
                                    h * r.oh + col) = O[t][p];
                        }
                }
            } else {
                sk.load(next, left, k4);
                sv.load(next, left, v4);
            }
            S.scale(gc);
#pragma unroll
            for (int s = 0; s < kTT; ++s)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int row = 16 * s + 4 * g + x;
                    const float w = weight[row + C - count];
#pragma unroll
                    for (int a = 0; a < State<T, D>::kTiles; ++a) {
                        const float kt = fk[row * G::kStride + 16 * a + l];
#pragma unroll
                        for (int p = 0; p < 2; ++p)
                            S.s[a][p] = mfma(kt, vf[s][p][x] * w, S.s[a][p]);
                    }
                }
        }
        n = next;
    }
    if (kNorm) S.scale(pow2(-exp_s));  // |exp_s| <= 120
    if constexpr (OUT) {
        // tokens past the sequence's end
        const int from = max(begin, len), to = (int)min((int64_t)begin + c.seg_len, (int64_t)c.T);
        for (int64_t i = tid; i < (int64_t)(to - from) * (dv / 8); i += G::kThreads) {
            const int64_t o = (int64_t)(from + i / (dv / 8)) * r.ot + b * r.ob + h * r.oh +
                              i % (dv / 8) * 8;
            if (kHalf && !r.o_f32) {
                *reinterpret_cast<u32x4 *>(static_cast<T *>(r.o) + o) = u32x4{0, 0, 0, 0};
            } else {
                u32x4 *z = reinterpret_cast<u32x4 *>(static_cast<float *>(r.o) + o);
                z[0] = z[1] = u32x4{0, 0, 0, 0};
            }
        }
        if (r.final_state && seg + 1 == c.segs) S.store(r.final_state + at, dk, dv);
    } else {
        S.store(r.slot + (int64_t)(seg + 1) * r.slot_seg + at, dk, dv);
    }
}

// Segments' own states into the states they start from, in place: slot s + 1
// holds segment s's own, slot 0 receives the initial one.
__global__ __launch_bounds__(256) void segment_states_kernel(LaCall c) {
    const LaRole &r = c.role[blockIdx.z];
    const int bh = blockIdx.y, e = blockIdx.x * 256 + threadIdx.x;
    const int size = r.dk * r.dv;
    if (e >= size) return;
    const int len = c.lens ? min(max(c.lens[bh / c.H], 0), c.T) : c.T;
    const float g = c.decay[bh % c.H], full = decay_power(g, c.seg_len);
    float *slot = r.slot + (int64_t)bh * size + e;
    float x = 0.f;
    if (r.init) {
        const int i = e / r.dv, j = e % r.dv;
        x = r.init[(int64_t)bh * size + (r.trans ? j * r.dk + i : e)];
    }
    slot[0] = x;
    for (int s = 0; s + 1 < c.segs; ++s) {
        const int tokens = min(max(len - s * c.seg_len, 0), c.seg_len);
        const float f = tokens == c.seg_len ? full : decay_power(g, tokens);
        x = __builtin_fmaf(f, x, slot[(s + 1) * r.slot_seg]);
        slot[(s + 1) * r.slot_seg] = x;
    }
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

template <typename T>
__device__ inline float load_value(const LaOperand &x, int t, int b, int h, int i) {
    return (float)static_cast<const T *>(
        x.p)[t * x.st + b * x.sb + (int64_t)(h / x.share) * x.sh + i];
}

// One token of every request, one workgroup each and head; thread j has column
// j of the state.
template <typename T>
__global__ __launch_bounds__(kLaMaxD) void linattn_step_kernel(LaStep c) {
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

template <typename T, int D>
void launch_chunks(const LaCall &c, bool out, hipStream_t s) {
    const int segs = out ? c.segs : c.segs - 1;
    LaCall k = c;
    if (!out) k.segs = segs;
    const int grid = c.roles * c.B * c.H * segs;
    if (out) linattn_kernel<T, D, true><<<grid, 2 * D, 0, s>>>(k);
    else linattn_kernel<T, D, false><<<grid, 2 * D, 0, s>>>(k);
}

void launch_by_type(const LaCall &c, bool out, int dtype, bool wide, hipStream_t s) {
    switch (dtype) {
        case SNN_F32:
            wide ? launch_chunks<float, 128>(c, out, s) : launch_chunks<float, 64>(c, out, s);
            break;
        case SNN_F16:
            wide ? launch_chunks<half_t, 128>(c, out, s) : launch_chunks<half_t, 64>(c, out, s);
            break;
        default:
            wide ? launch_chunks<bf16_t, 128>(c, out, s) : launch_chunks<bf16_t, 64>(c, out, s);
    }
}

}  // namespace

// Segments that fill the device: a launch should have about four workgroups of
// 128 head values, or eight of 64, for each compute unit; a segment has at least
// four chunks.
LaPlan linattn_plan(int T, int64_t heads, int roles, int width) {
    const int64_t want = (width > 64 ? 2 : 4) * kPlanCus;
    const int64_t have = std::max<int64_t>(heads * roles, 1);
    int64_t segs = std::min<int64_t>((want + have - 1) / have, T / 256);
    LaPlan p;
    p.segs = 1;
    p.seg_len = std::max(T, 1);
    if (segs > 1) {
        p.seg_len = (int)(((T + segs - 1) / segs + 63) / 64 * 64);
        p.segs = (T + p.seg_len - 1) / p.seg_len;
    }
    return p;
}

hipError_t launch_linattn(const LaCall &c, int dtype, hipStream_t s) {
    const bool wide = std::max(c.role[0].dk, c.role[0].dv) > 64;
    if (c.segs == 1) {
        launch_by_type(c, true, dtype, wide, s);
        return hipGetLastError();
    }
    // the roles that own slots
    LaCall own = c;
    own.roles = 0;
    for (int i = 0; i < c.roles; ++i)
        if (c.role[i].slot) own.role[own.roles++] = c.role[i];
    launch_by_type(own, false, dtype, wide, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int size = own.role[0].dk * own.role[0].dv;
    segment_states_kernel<<<dim3((size + 255) / 256, c.B * c.H, own.roles), 256, 0, s>>>(own);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    LaCall out = c;
    for (int i = 0; i < c.roles; ++i) {
        LaRole &r = out.role[i];
        const LaRole &from = r.slot ? r : c.role[r.slot_of];
        r.init = from.slot;
        r.init_seg = from.slot_seg;
        r.trans = r.slot ? 0 : 1;
    }
    launch_by_type(out, true, dtype, wide, s);
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
        case SNN_F32: linattn_step_kernel<float><<<grid, kLaMaxD, 0, s>>>(c); break;
        case SNN_F16: linattn_step_kernel<half_t><<<grid, kLaMaxD, 0, s>>>(c); break;
        default: linattn_step_kernel<bf16_t><<<grid, kLaMaxD, 0, s>>>(c); break;
    }
    return hipGetLastError();
}

}  // namespace snn
