// Linear attention with a decay per head (include/snn.h, "leaky sequence
// block"): S_t = g S_{t-1} + k_t^T v_t, o_t = scale q_t S_t.
//
// The gradients are the same recurrence with its operands exchanged (dq: q' =
// do, k' = v, v' = k, state S^T; dk: time reversed, q' = v, k' = do, v' = q,
// state R^T; dv: time reversed, q' = k, k' = q, v' = do, state R), so one
// kernel computes forward and backward; a launch runs up to kLaRoles of them.
//
// Whole sequences go in chunks of C = 32 tokens with the state between them,
// all of it on the matrix cores:
//   o_i = rs (sum_{j<=i} g^{i-j} ws (q_i.k_j) v_j + g^{i+first} q_i X)
//   X'  = g^C X + sum_j g^{C-first-j} ws k_j^T v_j
// A wave owns 16 or 32 columns of v and the state's columns with them, in registers,
// so waves exchange nothing but the staged tiles of q, k and v; each computes the
// chunk's scores q.k for itself (12 % of its matrix instructions at d = 128 with 32
// columns, 20 % at 64; in fp32 25 and 39 %).  Every product is arranged so that a
// result lies in the registers as the next product's operand: scores and output are
// taken transposed (s x t, dv x t), and the 16 rows of a result tile are the k values
// 4 g + r that lane group g holds of an operand, in whatever order, as long as both
// operands agree.
//
// 16-bit operands multiply exactly into fp32.  What is fp32 and becomes an
// operand is split: scores and state into two 16-bit parts (2^-16 of a term,
// far under the result's own rounding; one part would raise a bf16 result's
// error by up to 1.4), v g^j in the state's update into as many as keep fp32's
// precision (three bf16, two fp16).  fp16 parts are taken after a scaling by a
// power of two that puts the largest value near 2^14, so neither large sums nor
// small ones leave the type's range: the largest of a token's scores, of a column of
// the state, of a chunk's column of v g^j.  Two parts then end at 2^-39 of it.  (Shared
// by more than one token or column, a scale would let one take another's digits.  Two
// bf16 parts of every fp16 operand need no scales, but 180 matrix instructions a chunk
// in place of 84: 128 heads of 128 there and back 444 us against 370.)  fp32 operands go through the fp32
// matrix instructions as they are.
//
// A masked score is replaced by zero, but a zero times a later token's infinite
// or NaN value would still reach earlier outputs: where a chunk's v holds
// one, its tokens go one at a time.
//
// Few heads: the tokens are cut into segments, a first launch takes every
// segment's own state, a second adds them up (decayed; up to eight, each
// segment's workgroup adds those before it itself), a last computes the outputs
// from each segment's state.
//
// Measured: 32768 tokens of 16 heads of 128 (bf16) 221 us, traced as 71 + 14 + 141
// (own states, their sums, outputs), 2.4 TB/s of the least traffic; the outputs'
// kernel moves 4 TB/s.  Counters there: the matrix cores are busy in 51 % of its
// time, vector instructions take 31 %, and the two waves of a SIMD wait for memory
// or LDS in 29 % of theirs.  fp32 is bound by the fp32 matrix instructions: 512
// tokens of 256 heads of 64, forward and backward, 193 us; they take 63 % of the
// forward's outputs and 74 % of the backward.  fp16 of 64 (8 x 1000 tokens of 16
// heads, 33 us) is bound by the vector unit: 61 %, matrix cores 14 %.
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

// Up to this many segments each adds the states of those before it by itself
// rather than in a launch between (2000 tokens in 8 segments, 64 bf16 heads of 128:
// 69 against 74 us, 128 fp16 heads of 64: 57 against 61).  Beyond that a prompt still
// gains (in 16, 64 bf16 heads of 64: 34 against 37) and training loses (12 heads of
// 128, 4096 tokens: 130 against 115).
constexpr int kSumHere = 8;

// decay^e, e >= 0, by repeated squaring in fp64 (0^0 = 1)
__device__ inline float decay_power(float g, int e) {
    double r = 1.0, b = g;
    for (; e; e >>= 1, b *= b)
        if (e & 1) r *= b;
    return (float)r;
}

// n / d of uniform 0 <= n < 2^31 by 1 / d in fp64, which is exact: n + 1/2 is never
// within an error of a multiple of d.  An integer division takes ten times the
// instructions.
__device__ inline int divided(int n, double by) {
    return __builtin_amdgcn_readfirstlane((int)((n + 0.5) * by));
}
__device__ inline float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// largest over lanes l, l + 16, l + 32 and l + 48 of values >= 0: those that hold one
// token of the scores, or one column of the state
__device__ inline float column_max(float x) {
    const uint32_t a = __float_as_uint(x);
    const auto b = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const uint32_t m = __float_as_uint(fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1])));
    const auto c = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return fmaxf(__uint_as_float(c[0]), __uint_as_float(c[1]));
}
// m = max(m, |a|, |b|), NaN ignored: one instruction, where fmaxf would first quiet
// each operand
__device__ inline void grow(float &m, float a, float b) {
    asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(m) : "v"(a), "v"(b));
}
__device__ inline void grow_finite(float &m, float a) {
    a = __builtin_fabsf(a);
    if (a < __builtin_inff()) m = fmaxf(m, a);
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

// two values as 16 bits each (to nearest), the first in the low half
template <typename T>
__device__ inline uint32_t pack2(float x, float y) {
    typedef T T2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), T2));
}
template <typename T>
__device__ inline float low(uint32_t p) {
    if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(p << 16);
    else return (float)__builtin_bit_cast(half_t, (uint16_t)p);
}
template <typename T>
__device__ inline float high(uint32_t p) {
    if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(p & 0xffff0000u);
    else return (float)__builtin_bit_cast(half_t, (uint16_t)(p >> 16));
}
template <typename T>
__device__ inline u32x4 pack(const f32x4 &a, const f32x4 &b) {
    return u32x4{pack2<T>(a[0], a[1]), pack2<T>(a[2], a[3]), pack2<T>(b[0], b[1]),
                 pack2<T>(b[2], b[3])};
}
// The next part of a and b: their nearest 16-bit values, taken off them.  For bf16
// that is exact on the matrix cores too, with rows of -1 for the first four of the
// 8 and the last: two instructions of 16 cycles where the vector unit takes sixteen
// of 4 (training of 128 heads of 128 331 us against 338).
template <typename T>
__device__ inline u32x4 take_part(f32x4 &a, f32x4 &b, const u32x4 (&minus)[2]) {
    const u32x4 p = pack<T>(a, b);
    if constexpr (std::is_same_v<T, bf16_t>) {
        a = mfma<T>(minus[0], p, a);
        b = mfma<T>(minus[1], p, b);
    } else {
        a -= f32x4{low<T>(p[0]), high<T>(p[0]), low<T>(p[1]), high<T>(p[1])};
        b -= f32x4{low<T>(p[2]), high<T>(p[2]), low<T>(p[3]), high<T>(p[3])};
    }
    return p;
}
template <typename T>
__device__ inline void unpack(const u32x4 &p, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[2 * j] = low<T>(p[j]), x[2 * j + 1] = high<T>(p[j]);
}

// ---- geometry ----------------------------------------------------------------------
// D: head sizes up to 64 or 128, padded with zeros.  N: columns of a wave, one tile
// or a pair, so D / N waves make a workgroup.
//
// Of 64, a wave takes 16: the registers then hold four waves of a SIMD, with chunks of
// 32 tokens, instead of two with 32 columns and chunks of 64 (2000 tokens of 128 heads
// there and back: bf16 145 us against 169, fp16 172 against 175, now 168; 512 tokens of
// 256 fp32 heads 195 against 213).  Of 128 they do not: 16 while each workgroup has a
// compute unit to itself (101 tokens of 8 heads there and back: bf16 27 us against 30;
// of 30 fp32 heads 55 against 61), else 32, which compute the scores half as often
// (2000 tokens of 128 bf16 heads 316 against 344, 512 of 256 fp32 heads 512 against
// 596, with 13 registers a lane of the fp32 outputs' kernel in scratch).
template <typename T, int D, int N>
struct Geo {
    static constexpr bool kHalf = sizeof(T) == 2;
    // Tokens of a chunk (64 spill at d = 128: 512 x 16 tokens and heads took 174 us
    // against 142).
    static constexpr int C = 32;
    static constexpr int kPairs = N / 16, kWaves = D / N, kThreads = 64 * kWaves;
    static constexpr int kEu = D > 64 ? 2 : 4;  // waves of a SIMD at least
    // fp32: tiles of the head that a product takes together, for independent sums (at
    // 128 others run meanwhile, and one leaves less padding)
    static constexpr int kStep = D > 64 ? 1 : 2;
    static constexpr int kRun = 16 / sizeof(T);       // values of a 16-byte run
    static constexpr int kRuns = D / kRun;            // runs of a row
    static constexpr int kRows = kThreads / kRuns;    // rows that the threads stage at once
    static constexpr int kVec = C / kRows;            // runs a thread stages
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
template <typename T, int D, int N>
struct Source {
    const T *lane;  // this thread's run in the first row it stages of the next chunk
    int64_t step;
    bool live;      // the run lies within the head
    bool whole;     // the head fills the row
    __device__ inline void init(const LaOperand &x, int b, int h, int width, int last, int begin) {
        typedef Geo<T, D, N> G;
        const int run = threadIdx.x % G::kRuns, row = threadIdx.x / G::kRuns;
        step = last >= 0 ? -x.st : x.st;
        lane = static_cast<const T *>(x.p) + b * x.sb + (int64_t)divided(h, x.by_share) * x.sh +
               (last >= 0 ? last * x.st : 0) + (begin + row) * step + run * G::kRun;
        live = run * G::kRun < width;
        whole = width == D;
    }
    // the next `count` tokens, zeros past them and past the head
    __device__ inline void load(int count, u32x4 (&v)[Geo<T, D, N>::kVec]) const {
        typedef Geo<T, D, N> G;
        if (whole && count >= G::C) {
#pragma unroll
            for (int i = 0; i < G::kVec; ++i)
                v[i] = *reinterpret_cast<const u32x4 *>(lane + i * G::kRows * step);
        } else {
            const int row = threadIdx.x / G::kRuns;
#pragma unroll
            for (int i = 0; i < G::kVec; ++i) {
                v[i] = u32x4{0, 0, 0, 0};
                if (live && row + i * G::kRows < count)
                    v[i] = *reinterpret_cast<const u32x4 *>(lane + i * G::kRows * step);
            }
        }
    }
    __device__ inline void advance(int tokens) { lane += tokens * step; }
    __device__ static inline void stage(T *tile, const u32x4 (&v)[Geo<T, D, N>::kVec]) {
        typedef Geo<T, D, N> G;
        const int run = threadIdx.x % G::kRuns, row = threadIdx.x / G::kRuns;
#pragma unroll
        for (int i = 0; i < G::kVec; ++i)
            *reinterpret_cast<u32x4 *>(tile + G::at(row + i * G::kRows, run)) = v[i];
    }
};

// whether a staged run holds an infinity or NaN
template <typename T, int N>
__device__ inline bool not_finite(const u32x4 (&v)[N]) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
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

// 8 values of one column of column tile c, rows 4 g .. + 3 and 16 + 4 g .. + 3 of a
// row-major tile: within 16 lanes, the transposing read hands lane i element e of
// lane 4 e + i / 4's 4-value run (position i % 4), so lane L points at row 4 g + L / 4
// and the run of lanes 4 (L % 4) .. + 3.  Of 32 columns the even tile holds
// 8 (i / 4) + i % 4, the odd one those + 4: a lane's results of both are 8 neighbours
// in memory.
template <typename T, int D>
__device__ inline u32x4 read_columns(const T *tile, int c) {
    typedef Geo<T, D, 32> G;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int lane = threadIdx.x & 63, g = lane >> 4, L = lane & 15;
    const int row = 4 * g + (L >> 2);
    const T *a = tile + G::at(row, 4 * (c >> 1) + (L & 3)) + 4 * (c & 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(a + 16 * G::kStride));
    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
    return u32x4{x[0], x[1], y[0], y[1]};
}

// The state's columns of one wave: tile (a, p) holds rows row(a) + r and column
// col(p), r = 0 .. 3.
template <typename T, int D, int N>
struct State {
    static constexpr int kTiles = D / 16, kPairs = N / 16;
    f32x4 s[kTiles][kPairs];
    __device__ static inline int row(int a, int lane) {
        const int g = lane >> 4;
        return sizeof(T) == 2 ? 32 * (a >> 1) + 8 * g + 4 * (a & 1) : 16 * a + 4 * g;
    }
    __device__ static inline int col(int p, int w, int lane) {
        const int i = lane & 15, c = kPairs * w + p;
        return sizeof(T) == 2 ? 32 * (c >> 1) + 8 * (i >> 2) + 4 * (c & 1) + (i & 3) : 16 * c + i;
    }
    __device__ static inline int row(int a) { return row(a, threadIdx.x & 63); }
    __device__ static inline int col(int p) { return col(p, threadIdx.x >> 6, threadIdx.x & 63); }
    // from and to [dk][dv] (trans: [dv][dk]) in memory; what is out of range is
    // read as row 0, column 0 and dropped, so that no branch holds a load back
    __device__ inline void load(const float *from, bool trans, int dk, int dv) {
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < kPairs; ++p) s[a][p] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!from) return;
        if (trans) {
#pragma unroll
            for (int a = 0; a < kTiles; ++a)
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    const bool in = row(a) < dk && col(p) < dv;
                    s[a][p] = *reinterpret_cast<const f32x4 *>(
                        from + (in ? col(p) * dk + row(a) : 0));
                }
        } else {
#pragma unroll
            for (int a = 0; a < kTiles; ++a)
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    const float *x = from + (row(a) < dk && col(p) < dv ? row(a) * dv + col(p) : 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[a][p][r] = x[r * dv];
                }
        }
        if (dk < D || dv < D)
#pragma unroll
            for (int a = 0; a < kTiles; ++a)
#pragma unroll
                for (int p = 0; p < kPairs; ++p)
                    if (row(a) >= dk || col(p) >= dv) s[a][p] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ inline void store(float *to, int dk, int dv) const {
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < kPairs; ++p)
                if (row(a) < dk && col(p) < dv) {
                    float *x = to + row(a) * dv + col(p);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r * dv] = s[a][p][r];
                }
    }
    // Segment states between launches: a wave's tiles as they lie in its registers,
    // 16 bytes per lane.
    static constexpr int kSlot = D * D;
    __device__ static inline f32x4 *own(float *slot, int a, int p) {
        return reinterpret_cast<f32x4 *>(slot) +
               (((threadIdx.x >> 6) * kTiles + a) * kPairs + p) * 64 + (threadIdx.x & 63);
    }
    __device__ inline void store_slot(float *slot) const {
#pragma unroll
        for (int a = 0; a < kTiles; ++a)
#pragma unroll
            for (int p = 0; p < kPairs; ++p) *own(slot, a, p) = s[a][p];
    }
    // s = f s + the slot (trans: of a role whose state is this one transposed)
    __device__ inline void add_slot(float f, float *slot, bool trans) {
        if (trans) {
            // row col(p) and columns row(a) .. + 3 of the slot's state: row tile kPairs w + p,
            // column tile a, lanes 16 (l / 4) + 4 g .. + 3
            const int w = threadIdx.x >> 6, g = (threadIdx.x & 63) >> 4, l = threadIdx.x & 15;
            const float *from = slot + 256 * kPairs * kPairs * w + 64 * (l >> 2) + 16 * g + (l & 3);
#pragma unroll
            for (int a = 0; a < kTiles; ++a)
#pragma unroll
                for (int p = 0; p < kPairs; ++p)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[a][p][r] = __builtin_fmaf(
                            f, s[a][p][r],
                            from[256 * (kTiles * (a / kPairs * kPairs) + kPairs * p + a % kPairs) +
                                 4 * r]);
        } else {
#pragma unroll
            for (int a = 0; a < kTiles; ++a)
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    const f32x4 x = *own(slot, a, p);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[a][p][r] = __builtin_fmaf(f, s[a][p][r], x[r]);
                }
        }
    }
    __device__ inline void scale(int p, float f) {
#pragma unroll
        for (int a = 0; a < kTiles; ++a) s[a][p] *= f;
    }
    __device__ inline void scale(float f) {
#pragma unroll
        for (int p = 0; p < kPairs; ++p) scale(p, f);
    }
    // each column's largest finite magnitude
    __device__ inline void largest(float (&m)[kPairs]) const {
        bool bad = false;
#pragma unroll
        for (int p = 0; p < kPairs; ++p) {
            float x[2] = {};
#pragma unroll
            for (int a = 0; a < kTiles; ++a) {
                grow(x[0], s[a][p][0], s[a][p][1]);
                grow(x[1], s[a][p][2], s[a][p][3]);
            }
            m[p] = column_max(fmaxf(x[0], x[1]));
            bad |= !(m[p] < __builtin_inff());
        }
        if (!__any(bad)) return;
#pragma unroll
        for (int p = 0; p < kPairs; ++p) {
            m[p] = 0.f;
#pragma unroll
            for (int a = 0; a < kTiles; ++a)
#pragma unroll
                for (int r = 0; r < 4; ++r) grow_finite(m[p], s[a][p][r]);
            m[p] = column_max(m[p]);
        }
    }
};

// One workgroup: one role, sequence, head and segment.  OUT: outputs (and the
// final state); else the segment's own state alone, into its slot.
template <typename T, int D, int N, bool OUT>
__global__ __launch_bounds__((Geo<T, D, N>::kThreads), (Geo<T, D, N>::kEu))
void linattn_kernel(LaCall c) {
    typedef Geo<T, D, N> G;
    constexpr int C = G::C, kTT = C / 16;  // tiles of 16 tokens
    static_assert(kTT == 2);
    constexpr bool kHalf = G::kHalf, kNorm = std::is_same_v<T, half_t>;
    __shared__ __attribute__((aligned(16))) T tq[OUT ? G::kTile : 8], tk[G::kTile], tv[G::kTile];
    __shared__ float pw[C + 1];       // decay^i
    __shared__ float weight[2 * C];   // ws decay^(C - first - x), zero from x = C on
    __shared__ float score[48];       // rs ws decay^(x - 16)
    __shared__ int flag[2];

    const int item = xcd_local_item();
    const int unit = divided(item, c.by_roles), bh = divided(unit, c.by_segs);
    const int seg = unit - bh * c.segs, b = divided(bh, c.by_heads), h = bh - b * c.H;
    const LaRole r = c.role[item - unit * c.roles];
    // every line of the arguments on its way at once
    asm volatile("" ::"s"(r.q.p), "s"(r.k.st), "s"(r.v.p), "s"(r.v.by_share), "s"(r.o),
                 "s"(r.o_f32), "s"(r.final_state), "s"(r.rs), "s"(r.slot), "s"(r.slot_trans),
                 "s"(c.decay), "s"(c.T), "s"(c.segs));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 15, g = lane >> 4;
    const int len = c.lens ? min(max(c.lens[b], 0), c.T) : c.T;
    const int begin = seg * c.seg_len, end = (int)min((int64_t)begin + c.seg_len, (int64_t)len);
    const int dk = r.dk, dv = r.dv;
    const float decay = c.decay[h];
    Source<T, D, N> sq, sk, sv;
    const int last = r.reverse ? len - 1 : -1;  // len 0: no token is read
    if (OUT) sq.init(r.q, b, h, dk, last, begin);
    sk.init(r.k, b, h, dk, last, begin);
    sv.init(r.v, b, h, dv, last, begin);
    u32x4 q4[G::kVec], k4[G::kVec], v4[G::kVec];
    if (OUT) sq.load(end - begin, q4);
    sk.load(end - begin, k4);
    sv.load(end - begin, v4);

    static_assert(C < G::kThreads);
    if (tid <= C) pw[tid] = decay_power(decay, tid);
    if (tid < 2) flag[tid] = 0;

    State<T, D, N> S;
    const int64_t at = (int64_t)bh * dk * dv;
    // the state that enters this segment: the first one's is given; another's is in
    // its slot, or (few segments) the sum of those before it
    const int64_t slot_seg = (int64_t)c.B * c.H * State<T, D, N>::kSlot;
    float *slot = r.slot + (int64_t)bh * State<T, D, N>::kSlot;
    const bool ready = c.summed && (seg > 0 || c.copied);
    S.load(OUT && r.init && !ready ? r.init + at : nullptr, r.trans, dk, dv);
    if (OUT && c.segs > 1) {
        if (ready) S.add_slot(0.f, slot + seg * slot_seg, r.slot_trans);
        else
            for (int s = 0; s < seg; ++s)
                S.add_slot(decay_power(decay, min(max(len - s * c.seg_len, 0), c.seg_len)),
                           slot + (s + 1) * slot_seg, r.slot_trans);
    }
    int exp_s[G::kPairs] = {};  // fp16: column p of the state is s 2^-exp_s[p]

    // this lane's token and columns of the output, and their step over tokens
    const int64_t ostep = r.reverse ? -r.ot : r.ot;
    const bool o_f32 = r.o_f32;
    const int tile0 = G::kPairs * wave;  // its first tile of 16 columns
    const int ocol = kHalf ? 32 * (tile0 >> 1) + 4 * (tile0 & 1) + 8 * g : N * wave + 4 * g;
    char *out = static_cast<char *>(r.o) +
                (b * r.ob + h * r.oh + (r.reverse ? (len - 1) * r.ot : 0) + (begin + l) * ostep +
                 ocol) * (int64_t)(o_f32 ? 4 : sizeof(T));
    const int64_t obytes = ostep * (o_f32 ? 4 : sizeof(T));

    __syncthreads();
    for (int i = tid; i < 2 * C; i += G::kThreads)
        weight[i] = i < C ? r.ws * pw[max(C - r.first - i, 0)] : 0.f;
    if (tid < 48) score[tid] = r.rs * r.ws * pw[max(tid - 16, 0)];
    float tile[kTT];  // decays from tile to tile of 16 tokens
#pragma unroll
    for (int t = 0; t < kTT; ++t)
        tile[t] = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(pw[16 * t])));
    const float row = r.rs * pw[l] * (r.first ? decay : 1.f);

    const bool keep = r.final_state && seg + 1 == c.segs;  // the last chunk's state is used
    // -1 where a lane's row is the first four's, or the last four's, of 8 values
    u32x4 minus[2] = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (l == 4 * g + j)
            minus[0][j >> 1] = minus[1][2 + (j >> 1)] = j & 1 ? 0xbf800000u : 0xbf80u;
    int par = 0;
    for (int n = begin; n < end; par ^= 1) {
        int count = min(C, end - n);
        __syncthreads();  // the previous chunk's reads are done
        if (OUT) Source<T, D, N>::stage(tq, q4);
        Source<T, D, N>::stage(tk, k4);
        Source<T, D, N>::stage(tv, v4);
        if (OUT && __any(not_finite<T, G::kVec>(v4)) && lane == 0) flag[par] = 1;
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
        if (OUT) sq.advance(count);
        sk.advance(count);
        sv.advance(count);
        if (OUT) sq.load(left, q4);  // the next chunk, on its way meanwhile
        sk.load(left, k4);
        sv.load(left, v4);
        float largest[G::kPairs] = {};
        if constexpr (kNorm) S.largest(largest);

        if constexpr (kHalf) {
            u32x4 vf[G::kPairs];
            if constexpr (OUT) {
                f32x4 O[kTT][G::kPairs], P[kTT][kTT];
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) O[t][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s <= t; ++s) P[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                int exp_x[G::kPairs] = {};  // of the state as an operand, a column each
                if constexpr (kNorm)
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p)
                        exp_x[p] = min(scale_to_half(largest[p]), 126 - exp_s[p]);
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
                    for (int p = 0; p < G::kPairs; ++p) {
                        f32x4 x = S.s[2 * q][p], y = S.s[2 * q + 1][p];
                        if constexpr (kNorm) x *= pow2(exp_x[p]), y *= pow2(exp_x[p]);
                        const u32x4 hi = take_part<T>(x, y, minus), lo = pack<T>(x, y);
#pragma unroll
                        for (int t = 0; t < kTT; ++t) {
                            O[t][p] = mfma<T>(lo, qf[t], O[t][p]);
                            O[t][p] = mfma<T>(hi, qf[t], O[t][p]);
                        }
                    }
                }
#pragma unroll
                for (int p = 0; p < G::kPairs; ++p) vf[p] = read_columns<T, D>(tv, tile0 + p);
                // a column of the state is a row of the output: lane 4 g + x has its scale
                if constexpr (kNorm)
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) {
                        const int own = __float_as_int(pow2(-(exp_x[p] + exp_s[p])));
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float back = __int_as_float(
                                __builtin_amdgcn_ds_bpermute(4 * (4 * g + x), own));
#pragma unroll
                            for (int t = 0; t < kTT; ++t) O[t][p][x] *= back;
                        }
                    }
                // scores: decayed, those of later tokens zero.  A tile's row is s = 4 g + x,
                // its column t = l, of the same 16 tokens or the 16 before
                float near[4], far[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    near[x] = score[16 + l - 4 * g - x];
                    far[x] = score[32 + l - 4 * g - x];
                }
                float most[kTT][2] = {};
#pragma unroll
                for (int t = 0; t < kTT; ++t)
#pragma unroll
                    for (int s = 0; s <= t; ++s) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            float e = P[t][s][x];
                            if (s == t) e = l - 4 * g - x >= 0 ? e * near[x] : 0.f;
                            else e *= far[x];
                            P[t][s][x] = e;
                        }
                        if constexpr (kNorm) {
                            grow(most[t][0], P[t][s][0], P[t][s][1]);
                            grow(most[t][1], P[t][s][2], P[t][s][3]);
                        }
                    }
                // a token's scores have a scale of their own: another token, a later one
                // least of all, must not take its digits.  At most 2^60: what smaller scores
                // lose is far below an fp16 output's least step
                int exp_p[kTT] = {};
                if constexpr (kNorm) {
                    float m[kTT];
#pragma unroll
                    for (int t = 0; t < kTT; ++t)
                        m[t] = column_max(fmaxf(most[t][0], most[t][1]));
                    if (__any(!(fmaxf(m[0], m[1]) < __builtin_inff()))) {
                        // of an infinite q or k: the finite ones'
#pragma unroll
                        for (int t = 0; t < kTT; ++t) {
                            m[t] = 0.f;
#pragma unroll
                            for (int s = 0; s <= t; ++s)
#pragma unroll
                                for (int x = 0; x < 4; ++x) grow_finite(m[t], P[t][s][x]);
                            m[t] = column_max(m[t]);
                        }
                    }
#pragma unroll
                    for (int t = 0; t < kTT; ++t) exp_p[t] = min(60, scale_to_half(m[t]));
                }
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
                    float f = row * tile[t];
                    if constexpr (kNorm) f = __builtin_ldexpf(f, exp_p[t]);
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) O[t][p] *= f;
                    f32x4 x = P[t][0], y = t ? P[t][t] : f32x4{0.f, 0.f, 0.f, 0.f};
                    if constexpr (kNorm) {
                        const float fp = pow2(exp_p[t]);
                        x *= fp, y *= fp;
                    }
                    const u32x4 hi = take_part<T>(x, y, minus), lo = pack<T>(x, y);
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) {
                        O[t][p] = mfma<T>(vf[p], lo, O[t][p]);
                        O[t][p] = mfma<T>(vf[p], hi, O[t][p]);
                    }
                    // token 16 t + l, columns 8 g .. 8 g + 7 of 32 or four of them
                    if (16 * t + l < count && ocol < dv) {
                        char *to = out + 16 * t * obytes;
                        if constexpr (kNorm)
#pragma unroll
                            for (int p = 0; p < G::kPairs; ++p) O[t][p] *= pow2(-exp_p[t]);
                        if (o_f32) {
#pragma unroll
                            for (int p = 0; p < G::kPairs; ++p)
                                reinterpret_cast<f32x4 *>(to)[p] = O[t][p];
                        } else {
                            u32x2 half[G::kPairs];
#pragma unroll
                            for (int p = 0; p < G::kPairs; ++p)
                                half[p] = u32x2{pack2<T>(O[t][p][0], O[t][p][1]),
                                                pack2<T>(O[t][p][2], O[t][p][3])};
                            if constexpr (G::kPairs == 2)
                                *reinterpret_cast<u32x4 *>(to) =
                                    u32x4{half[0][0], half[0][1], half[1][0], half[1][1]};
                            else *reinterpret_cast<u32x2 *>(to) = half[0];
                        }
                    }
                }
            } else {
#pragma unroll
                for (int p = 0; p < G::kPairs; ++p) vf[p] = read_columns<T, D>(tv, tile0 + p);
            }
            if (OUT && left <= 0 && !keep) break;
            // the state's update
            const float *wt = weight + (C - count) + 4 * g;
            auto weighted = [&](int p, float (&x)[8]) {
                unpack<T>(vf[p], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= wt[16 * (j >> 2) + (j & 3)];
            };
            float w[G::kPairs][8];
            if constexpr (kNorm) {
                float most[G::kPairs];
                bool bad = false;
#pragma unroll
                for (int p = 0; p < G::kPairs; ++p) {
                    float m[2] = {};
                    weighted(p, w[p]);
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        grow(m[0], w[p][j], w[p][j + 1]);
                        grow(m[1], w[p][j + 2], w[p][j + 3]);
                    }
                    most[p] = column_max(fmaxf(m[0], m[1]));
                    bad |= !(most[p] < __builtin_inff());
                }
                if (__any(bad)) {
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) {
                        most[p] = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) grow_finite(most[p], w[p][j]);
                        most[p] = column_max(most[p]);
                    }
                }
#pragma unroll
                for (int p = 0; p < G::kPairs; ++p) {
                    // the scale of this chunk's v g^j, unless the state would leave 2^61
                    int e = most[p] > 0.f ? scale_to_half(most[p]) : exp_s[p];
                    const float left_s = largest[p] * __builtin_fabsf(gc);
                    if (left_s > 0.f)
                        e = min(e, exp_s[p] + min(120, scale_to_half(left_s) + 46));
                    S.scale(p, left_s > 0.f ? __builtin_ldexpf(gc, e - exp_s[p]) : 0.f);
                    exp_s[p] = e;
                }
            } else {
                S.scale(gc);
            }
            constexpr int kParts = kNorm ? 2 : 3;
            u32x4 part[G::kPairs][kParts];
#pragma unroll
            for (int p = 0; p < G::kPairs; ++p) {
                float x[8];
                if constexpr (kNorm) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = w[p][j] * pow2(exp_s[p]);
                } else {
                    weighted(p, x);
                }
                f32x4 y = {x[0], x[1], x[2], x[3]}, z = {x[4], x[5], x[6], x[7]};
#pragma unroll
                for (int m = 0; m + 1 < kParts; ++m) part[p][m] = take_part<T>(y, z, minus);
                part[p][kParts - 1] = pack<T>(y, z);
            }
#pragma unroll
            for (int a = 0; a < State<T, D, N>::kTiles; ++a) {
                const u32x4 kt = read_columns<T, D>(tk, a);
#pragma unroll
                for (int m = kParts - 1; m >= 0; --m)
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p)
                        S.s[a][p] = mfma<T>(kt, part[p][m], S.s[a][p]);
            }
        } else if (N * wave < dv) {
            const float *fq = reinterpret_cast<const float *>(tq),
                        *fk = reinterpret_cast<const float *>(tk),
                        *fv = reinterpret_cast<const float *>(tv);
            f32x4 vf[kTT][G::kPairs];
            auto read_v = [&] {
#pragma unroll
                for (int s = 0; s < kTT; ++s)
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p)
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            vf[s][p][x] =
                                fv[(16 * s + 4 * g + x) * G::kStride + N * wave + 16 * p + l];
            };
            if constexpr (OUT) {
                f32x4 O[kTT][G::kPairs], P[kTT][kTT];
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) O[t][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s <= t; ++s) P[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int a = 0; a < State<T, D, N>::kTiles; ++a) {
                    if (a % G::kStep == 0 && 16 * a >= dk) break;  // nothing but padding from here
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
                            for (int p = 0; p < G::kPairs; ++p)
                                O[t][p] = mfma(S.s[a][p][x], qf[t][x], O[t][p]);
                        }
                }
                read_v();
                float near[4], far[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    near[x] = score[16 + l - 4 * g - x];
                    far[x] = score[32 + l - 4 * g - x];
                }
#pragma unroll
                for (int t = 0; t < kTT; ++t) {
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) O[t][p] *= row * tile[t];
#pragma unroll
                    for (int s = 0; s <= t; ++s)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            float e = P[t][s][x];
                            if (s == t) e = l - 4 * g - x >= 0 ? e * near[x] : 0.f;
                            else e *= far[x];
#pragma unroll
                            for (int p = 0; p < G::kPairs; ++p)
                                O[t][p] = mfma(vf[s][p][x], e, O[t][p]);
                        }
                    if (16 * t + l < count)
#pragma unroll
                        for (int p = 0; p < G::kPairs; ++p)
                            if (ocol + 16 * p < dv)
                                *reinterpret_cast<f32x4 *>(out + 16 * t * obytes + 64 * p) =
                                    O[t][p];
                }
            }
            if (!OUT) read_v();
            if (OUT && left <= 0 && !keep) break;
            S.scale(gc);
#pragma unroll
            for (int s = 0; s < kTT; ++s)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float w = weight[16 * s + 4 * g + x + C - count];
#pragma unroll
                    for (int p = 0; p < G::kPairs; ++p) vf[s][p][x] *= w;
                }
#pragma unroll
            for (int a0 = 0; a0 < State<T, D, N>::kTiles; a0 += G::kStep) {
                if (16 * a0 >= dk) break;
#pragma unroll
                for (int s = 0; s < kTT; ++s)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int a = a0; a < a0 + G::kStep; ++a) {
                            const float kt = fk[(16 * s + 4 * g + x) * G::kStride + 16 * a + l];
#pragma unroll
                            for (int p = 0; p < G::kPairs; ++p)
                                S.s[a][p] = mfma(kt, vf[s][p][x], S.s[a][p]);
                        }
            }
        }
        n = next;
        out += count * obytes;
    }
    if (kNorm)
#pragma unroll
        for (int p = 0; p < G::kPairs; ++p) S.scale(p, pow2(-exp_s[p]));  // |exp_s| <= 120
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
        if (keep) S.store(r.final_state + at, dk, dv);
    } else {
        S.store_slot(slot + (seg + 1) * slot_seg);
    }
}

// Segments' own states into the states they start from, in place: slot s + 1
// holds segment s's own, slot 0 receives the initial one where it is read from
// there.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void segment_states_kernel(LaCall c) {
    typedef State<T, D, N> St;
    const LaRole &r = c.role[blockIdx.z];
    // four rows of a column per thread, in the slots' order
    const int bh = blockIdx.y, e = blockIdx.x * 256 + threadIdx.x;
    const int tile = e >> 6, lane = e & 63, p = tile % St::kPairs,
              a = tile / St::kPairs % St::kTiles;
    const int i = St::row(a, lane), j = St::col(p, tile / St::kPairs / St::kTiles, lane);
    const int len = c.lens ? min(max(c.lens[bh / c.H], 0), c.T) : c.T;
    const float g = c.decay[bh % c.H], full = decay_power(g, c.seg_len);
    const int64_t slot_seg = (int64_t)c.B * c.H * (St::kSlot / 4);
    f32x4 *slot = reinterpret_cast<f32x4 *>(r.slot) + (int64_t)bh * (St::kSlot / 4) + e;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (r.init && i < r.dk && j < r.dv)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] = r.init[(int64_t)bh * r.dk * r.dv +
                          (r.trans ? j * r.dk + i + k : (i + k) * r.dv + j)];
    if (c.copied) slot[0] = x;
    constexpr int kAhead = 8;  // loads on their way together
    for (int s0 = 0; s0 + 1 < c.segs; s0 += kAhead) {
        f32x4 own[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (s0 + k + 1 < c.segs) own[k] = slot[(s0 + k + 1) * slot_seg];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int s = s0 + k;
            if (s + 1 >= c.segs) break;
            const int tokens = min(max(len - s * c.seg_len, 0), c.seg_len);
            const float f = tokens == c.seg_len ? full : decay_power(g, tokens);
#pragma unroll
            for (int m = 0; m < 4; ++m) x[m] = __builtin_fmaf(f, x[m], own[k][m]);
            slot[(s + 1) * slot_seg] = x;
        }
    }
}

// dst[t,b,hk,:] = sum over the group's heads of src[t,b,h,:] (fp32, ascending), for
// two tensors at once.  Bound by memory: two of 16384 tokens of 8 heads of 64 into 4 take
// 17 us in fp32, 5.9 TB/s (in a launch each 19).
template <typename T>
__global__ __launch_bounds__(256) void group_sum_kernel(LaGroupSum first, LaGroupSum second, int B,
                                                        int KV, int share, int64_t rows) {
    const LaGroupSum &c = blockIdx.y ? second : first;
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int d = c.d, d8 = d / 8;
    const int64_t y = x / d8;
    if (y >= rows) return;
    const int i = (int)(x - y * d8) * 8;
    const int64_t tb = y / KV, t = tb / B;
    const int hk = (int)(y - tb * KV);
    float s[8] = {};
    for (int m = 0; m < share; ++m) {
        const float *p = c.src + (y * share + m) * d + i;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += p[e];
    }
    T *o = static_cast<T *>(c.dst) + t * c.st + (tb - t * B) * c.sb + hk * c.sh + i;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (T)s[e];
}

template <typename T>
__device__ inline float load_value(const LaOperand &x, int t, int b, int h, int i) {
    return (float)static_cast<const T *>(
        x.p)[t * x.st + b * x.sb + (int64_t)divided(h, x.by_share) * x.sh + i];
}

// One token of every request.  The state is read and written once, 16 bytes per
// lane, and everything else is small: a workgroup takes a head's whole state, or
// (few requests) a slice of 32 or more of its columns, so that the loads of all
// states are on their way at once.  Thread (i, j) has rows i, i + rows, ... of
// columns 4 j .. 4 j + 3; the rows' shares of the output are added in order.
// 64 requests of 32 heads of 128 x 128: 57 us, 4.8 TB/s, a large copy's rate.
constexpr int kStepThreads = 256, kStepAhead = 8;

template <typename T>
__global__ __launch_bounds__(kStepThreads) void linattn_step_kernel(LaStep c) {
    __shared__ float qs[kLaMaxD], ks[kLaMaxD], part[kStepThreads * 4];
    const int tid = threadIdx.x;
    const int bh = divided(blockIdx.x, c.by_slices), slice = blockIdx.x - bh * c.slices;
    const int b = divided(bh, c.by_heads), h = bh - b * c.H;
    const int slot = c.slots ? c.slots[b] : b;
    const int col0 = slice * c.cols, cols = min(c.cols, c.dv - col0);
    T *o = static_cast<T *>(c.o) + b * c.ob + h * c.oh + col0;
    if (slot < 0 || slot >= c.n_slots) {  // idle
        if (tid < cols) o[tid] = (T)0.f;
        return;
    }
    const int quads = cols / 4, rows = kStepThreads / quads, i0 = tid / quads, j = tid % quads * 4;
    const bool live = i0 < rows;
    const int64_t at = ((int64_t)slot * c.H + h) * c.dk * c.dv + col0 + j;
    const float *in = c.in + at;
    float *out = c.out + at;
    f32x4 s[kStepAhead];
#pragma unroll
    for (int u = 0; u < kStepAhead; ++u)
        if (live && i0 + u * rows < c.dk)
            s[u] = *reinterpret_cast<const f32x4 *>(in + (int64_t)(i0 + u * rows) * c.dv);
    if (tid < c.dk) {
        qs[tid] = load_value<T>(c.q, 0, b, h, tid);
        ks[tid] = load_value<T>(c.k, 0, b, h, tid);
    }
    const float g = c.decay[h];
    f32x4 v = {0.f, 0.f, 0.f, 0.f}, sum = {0.f, 0.f, 0.f, 0.f};
    if (live)
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = load_value<T>(c.v, 0, b, h, col0 + j + x);
    __syncthreads();
    for (int i = i0; live && i < c.dk; i += kStepAhead * rows) {
        f32x4 next[kStepAhead];
#pragma unroll
        for (int u = 0; u < kStepAhead; ++u)
            if (i + (kStepAhead + u) * rows < c.dk)
                next[u] = *reinterpret_cast<const f32x4 *>(
                    in + (int64_t)(i + (kStepAhead + u) * rows) * c.dv);
#pragma unroll
        for (int u = 0; u < kStepAhead; ++u) {
            const int r = i + u * rows;
            if (r >= c.dk) continue;
            const float k = ks[r], q = qs[r];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                s[u][x] = __builtin_fmaf(k, v[x], s[u][x] * g);
                sum[x] = __builtin_fmaf(q, s[u][x], sum[x]);
            }
            *reinterpret_cast<f32x4 *>(out + (int64_t)r * c.dv) = s[u];
        }
#pragma unroll
        for (int u = 0; u < kStepAhead; ++u) s[u] = next[u];
    }
    if (live) *reinterpret_cast<f32x4 *>(part + i0 * cols + j) = sum;
    __syncthreads();
    if (tid < cols) {
        float t = 0.f;
        for (int r = 0; r < rows; ++r) t += part[r * cols + tid];
        o[tid] = (T)(t * c.scale);
    }
}

void set_divisors(LaCall &c) {
    c.by_roles = 1.0 / c.roles;
    c.by_segs = 1.0 / c.segs;
    c.by_heads = 1.0 / c.H;
}

template <typename T, int D, int N>
hipError_t launch_chunks(const LaCall &c, hipStream_t s) {
    LaCall out = c;
    set_divisors(out);
    if (c.segs > 1) {
        // the roles that own slots
        LaCall own = c;
        own.roles = 0;
        for (int i = 0; i < c.roles; ++i)
            if (!c.role[i].slot_trans) own.role[own.roles++] = c.role[i];
        own.segs = c.segs - 1;
        set_divisors(own);
        linattn_kernel<T, D, N, false>
            <<<own.roles * c.B * c.H * own.segs, Geo<T, D, N>::kThreads, 0, s>>>(own);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        // a final state written over the initial one must not reach the first
        // segment's start
        for (int i = 0; i < c.roles; ++i)
            out.copied |= c.role[i].init && c.role[i].init == c.role[i].final_state;
        out.summed = out.copied || c.segs > kSumHere;
        if (out.summed) {
            LaCall sum = out;
            sum.roles = own.roles;
            for (int i = 0; i < own.roles; ++i) sum.role[i] = own.role[i];
            segment_states_kernel<T, D, N>
                <<<dim3(D * D / 1024, c.B * c.H, own.roles), 256, 0, s>>>(sum);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    linattn_kernel<T, D, N, true>
        <<<c.roles * c.B * c.H * c.segs, Geo<T, D, N>::kThreads, 0, s>>>(out);
    return hipGetLastError();
}

}  // namespace

// As many segments of 128 tokens or more as the workgroups resident at once have room
// for: two of 128 head values on a compute unit, four of 64.  Bf16 training of 128
// heads of 128 (2048 tokens): the forward in 4 segments 130 us, in 2 149; the
// backward's 384 heads and roles uncut 276, in 2 283 (and with a short segment for the
// 128 slots left 282).  Fp32 of 256 heads of 64 (512 tokens): the forward in 4
// segments 70 us, in 3 85.
// While each has a compute unit to itself, shorter ones too: a chunk of 32 tokens in
// fp32 (30 heads of 128 there and back, 101 tokens: 53 us, uncut 74; 8 heads, 1000
// tokens: 98, in seven 135), 64 tokens in 16 bits from three on (the same in bf16,
// 1000 tokens: 58 against 59; 30 heads, 128 tokens in two 31, uncut 26).  Two fp32
// workgroups of 128 on a compute unit slow each other down, which three segments are
// worth (129 heads, 384 tokens: 89 us, uncut 110; 4096: 784 and 1165) and two only over
// long sequences (255 heads, 256 tokens: 89, uncut 80; 512: 156 and 157; 800: 229 and
// 242; 4096: 1075 and 1186).
LaPlan linattn_plan(int T, int64_t heads, int roles, int width, int dtype) {
    const int64_t slots = (width > 64 ? 2 : 4) * kPlanCus;
    const int64_t units = std::max<int64_t>(heads * roles, 1);
    const int least = dtype == SNN_F32 ? 32 : 64, most = (T - 1) / least + 1;
    int64_t segs = std::min<int64_t>(slots / units, T / 128);
    if (dtype == SNN_F32 && width > 64 && segs == 2 && 2 * units > kPlanCus && T < 768) segs = 1;
    if (dtype == SNN_F32 || most > 2)
        segs = std::max(segs, std::min<int64_t>(kPlanCus / units, most));
    LaPlan p;
    p.segs = 1;
    p.seg_len = std::max(T, 1);
    p.slot_bytes = 0;
    if (segs > 1) {
        p.seg_len = (int)(((T + segs - 1) / segs + least - 1) / least * least);
        p.segs = (T + p.seg_len - 1) / p.seg_len;
        if (p.segs > 1) {
            const size_t d = width > 64 ? 128 : 64;
            p.slot_bytes = align_up((size_t)p.segs * heads * d * d * sizeof(float));
        }
    }
    return p;
}

template <typename T>
static hipError_t launch_width(const LaCall &c, hipStream_t s) {
    if (std::max(c.role[0].dk, c.role[0].dv) <= 64) return launch_chunks<T, 64, 16>(c, s);
    return (int64_t)c.roles * c.B * c.H * c.segs <= kPlanCus ? launch_chunks<T, 128, 16>(c, s)
                                                             : launch_chunks<T, 128, 32>(c, s);
}

hipError_t launch_linattn(const LaCall &c, int dtype, hipStream_t s) {
    // more heads than one launch takes, uncut by far: a role each
    if (c.roles > 1 && (int64_t)c.roles * c.B * c.H >= kLaMaxGroups) {
        for (int i = 0; i < c.roles; ++i) {
            LaCall one = c;
            one.role[0] = c.role[i];
            one.roles = 1;
            const hipError_t e = launch_linattn(one, dtype, s);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    switch (dtype) {
        case SNN_F32: return launch_width<float>(c, s);
        case SNN_F16: return launch_width<half_t>(c, s);
        default: return launch_width<bf16_t>(c, s);
    }
}

hipError_t launch_group_sum(const LaGroupSum &a, const LaGroupSum &b, int T, int B, int KV,
                            int share, int dtype, hipStream_t s) {
    const int64_t rows = (int64_t)T * B * KV;
    const dim3 grid((unsigned)((rows * (std::max(a.d, b.d) / 8) + 255) / 256), 2);
    switch (dtype) {
        case SNN_F32: group_sum_kernel<float><<<grid, 256, 0, s>>>(a, b, B, KV, share, rows); break;
        case SNN_F16:
            group_sum_kernel<half_t><<<grid, 256, 0, s>>>(a, b, B, KV, share, rows);
            break;
        default: group_sum_kernel<bf16_t><<<grid, 256, 0, s>>>(a, b, B, KV, share, rows);
    }
    return hipGetLastError();
}

hipError_t launch_linattn_step(const LaStep &call, int B, int dtype, hipStream_t s) {
    LaStep c = call;
    // 64 requests of 32 heads of 128 x 128 fill the device uncut; one request's 16
    // heads of 64 x 64 take 32 workgroups of 32 columns
    c.cols = c.dv;
    while (c.cols % 64 == 0 && (int64_t)B * c.H * (c.dv / c.cols) < 4 * kPlanCus) c.cols /= 2;
    c.slices = c.dv / c.cols;
    c.by_slices = 1.0 / c.slices;
    c.by_heads = 1.0 / c.H;
    const int grid = B * c.H * c.slices;
    switch (dtype) {
        case SNN_F32: linattn_step_kernel<float><<<grid, kStepThreads, 0, s>>>(c); break;
        case SNN_F16: linattn_step_kernel<half_t><<<grid, kStepThreads, 0, s>>>(c); break;
        default: linattn_step_kernel<bf16_t><<<grid, kStepThreads, 0, s>>>(c); break;
    }
    return hipGetLastError();
}

}  // namespace snn
