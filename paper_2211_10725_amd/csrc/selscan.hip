// Selective scan: leaky integrators whose step the input chooses (include/snn.h,
// "selective leaky block").
//
//     h_t[i] = exp(d_t a[i]) h_{t-1}[i] + d_t u_t b_t[i],   y_t = c_t . h_t + skip u_t
//
// Every decay is a channel's and an integrator's own, so nothing here is a matrix
// product: a token costs each integrator an exponential (two issue slots) and four
// multiply-adds, and the vector unit bounds it, at 24 cycles for 64 lanes; 8 x 2048 tokens
// of 2048 channels of 16 integrators take at least 82 us forward and, with 11 slots more
// and the states computed again, 250 backward.  A lane is a channel, so that the two
// integrators it holds need no exchange between lanes; the halves of a wave and the waves
// of a workgroup hold further integrators of the same 32 channels (rounds of 16 where there
// are more).  16 tokens at a time: the workgroup stages their steps d and d u (one softplus
// for all of a channel's integrators) and b and c in LDS, the waves run through them, and
// what they add to each (token, channel) is summed over the halves by an exchange and over
// the waves through LDS, in order.
//
// At the sizes above (forward 216 us, backward 533) 512 workgroups of four waves leave a
// SIMD two waves, of two workgroups, one of which runs while the other stages a tile or
// adds up its sums (256 workgroups of 64 channels in eight waves: backward 592 us where
// these took 552; 512 x 16 tokens of 1024 channels in fp32 161 and 144).  Also tried:
// four integrators a lane in half as many waves (forward 256 against 228, backward 852 against
// 722 at that time); two buffers of staged tiles, the next one staged before the barrier
// (backward 632 against 610); a tile's values prepared before the last one is stored (1055:
// registers); three waves of a SIMD backward, a tile's values read from LDS twice (these
// sizes there and back 791 against 766, in fp32 230 against 202; four times as many
// sequences 2374 against 2598).
//
// Few channels and long sequences: the sequence is cut into segments.  A first pass
// leaves each segment's end state from a zero start and its sum of steps (over a
// segment the decay is exp(a sum d)), a second joins them, the third runs every segment
// from its true start: 16384 tokens of 2048 channels, bf16, 258 us, of which the first pass
// takes two fifths.
//
// Backward, tile by tile from the end: the forward left the states before each tile of
// 16 tokens, the tile's states and decays are computed again into registers, then
//     g_t = c_t gy_t + exp(d_{t+1} a) g_{t+1},   q = exp(d_t a) g_t h_{t-1},
//     dc_t += gy_t h_t, db_t += d u g_t (sums over channels), d(d u) = b_t . g_t,
//     d(d) += a q, da += d q.
// The sums over channels are sums over the lanes of a half: the 4 values of a token (2
// integrators of b and c) are halved twice by exchanges that leave each lane half of the
// values, and joined with those of 7 more tokens, two to three instructions for a value of 64
// lanes; the workgroups' sums are added by another kernel in order.  The sums over tokens,
// of da and of skip's and dt_bias' gradients, are chains of T / 16 additions of a segment or
// a sequence: a tile's terms are added up first, da's by themselves and the others by their
// 16 threads at the end.
#include <type_traits>

#include "block_common.hpp"

namespace snn {
namespace {

constexpr int kTile = kSelscanTile;  // tokens
constexpr int kLanes = 64;
constexpr int kChans = 32;           // channels of a workgroup, and of half a wave
constexpr int H = 2;                 // integrators of a lane
constexpr int kSlots = 2 * H;        // their values of b and c for a token

// Where this workgroup works.
struct Place {
    int tile, seg, b, g, c0, live;  // channel tile, .., first channel, channels
};
__device__ inline Place place_of(const Selscan &a, int segs) {
    Place p;
    int x = xcd_local_item();  // neighbours share lines of 64 channels: on one XCD
    p.tile = x % a.tiles;
    x /= a.tiles;
    p.seg = x % segs;
    p.b = x / segs;
    const int per = a.tiles / a.groups, k = p.tile % per;
    p.g = p.tile / per;
    const int size = a.n / a.groups;
    p.c0 = p.g * size + k * kChans;
    p.live = min(kChans, size - k * kChans);
    return p;
}

__device__ inline int length_of(const Selscan &a, int b) {
    return a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
}

// A thread's place in a tensor: its token of the segment's first tile, and from there on
// whole tiles, which the scalar unit multiplies out.
template <typename T>
struct Walk {
    T *at;
    int64_t step;
    __device__ inline T *tile(int tokens) const { return at + tokens * step; }
};
template <typename T>
__device__ inline Walk<T> walk_rows(const SelscanRows &x, int t, const Place &p, int se) {
    return {static_cast<T *>(const_cast<void *>(x.p)) + t * x.st + p.b * x.sb + p.c0 + se, x.st};
}
template <typename T>
__device__ inline Walk<T> walk_vec(const SelscanVec &x, int t, const Place &p, int i) {
    return {static_cast<T *>(const_cast<void *>(x.p)) + t * x.st + p.b * x.sb + p.g * x.sg + i,
            x.st};
}
// EL values of a row, all of a workgroup's channels there or only m of these
template <typename T, int EL>
__device__ inline void fetch_run(Raw<T, EL> &r, const T *at, const Place &p, int m) {
    if (p.live == kChans) __builtin_memcpy(r.w, at, sizeof(r.w));
    else r.load(at, m);
}
template <typename T, int EL>
__device__ inline void put_run(T *at, const Place &p, int m, const float (&v)[EL]) {
    store_run(at, p.live == kChans ? EL : m, v);
}

// a log2 e, finite for every finite a: times a step of 0, as past a sequence, it has to be 0
__device__ inline float rate(float a) {
    const float x = a * kLog2e;
    return __builtin_fabsf(x) > __FLT_MAX__ ? __builtin_copysignf(__FLT_MAX__, x) : x;
}

// raw steps and their bias to steps, the condition outside the loop: one stretch of
// code in which the elements' chains overlap
template <int EL>
__device__ inline void steps(int soft, float (&d)[EL], const float (&bias)[EL]) {
#pragma unroll
    for (int j = 0; j < EL; ++j) d[j] += bias[j];
    if (soft)
#pragma unroll
        for (int j = 0; j < EL; ++j) {
            float slope;
            softplus(d[j], d[j], slope);
        }
}

// W waves, each with 2 H integrators of the 32 channels at once: H in each half.
template <int W>
struct Geo {
    static constexpr int kThreads = kLanes * W;
    static constexpr int kTok = 4 * W;           // threads that stage a token
    static constexpr int kEl = kChans / kTok;    // channels of such a thread
    static constexpr int kRow = 2 * H * W;       // integrators at once
};

// b and c of a tile for half a wave, 16 values to a register: token t's are the 2 H from
// 2 H t on.  Every lane wants the same ones; a register read with its lanes' own 16
// values (a quarter of the LDS traffic of a broadcast read) and the operand of an
// instruction that takes one lane of 16 for all of them.
constexpr int kVecRows = kTile * kSlots / 16;
using Vecs = float[kVecRows][16];

template <int N, int I = 0, typename F>
__device__ inline void each(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}
template <int L>
__device__ inline float lane_of16(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x150 + L, 0xf, 0xf, true));
}
// acc + (lane L of 16 of v) x.  The wait is for a v that the instruction before wrote; for
// the result see settle.
template <int L>
__device__ inline void fma_lane(float &acc, float v, float x) {
    asm("s_nop 1\n\tv_fmac_f32_dpp %0, %1, %2 row_newbcast:%3 row_mask:0xf bank_mask:0xf"
        : "+v"(acc)
        : "v"(v), "v"(x), "n"(L));
}
// g[k] += (lane L + H + k of 16 of v) x, and the sum over k of (lane L + k of v) g[k]
template <int L>
__device__ inline float fma_dot_lanes(float (&g)[H], float v, float x) {
    float r;
    asm("s_nop 1\n\t"
        "v_fmac_f32_dpp %0, %3, %4 row_newbcast:%7 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %1, %3, %4 row_newbcast:%8 row_mask:0xf bank_mask:0xf\n\t"
        "v_mul_f32_dpp %2, %3, %0 row_newbcast:%5 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %2, %3, %1 row_newbcast:%6 row_mask:0xf bank_mask:0xf"
        : "+&v"(g[0]), "+&v"(g[1]), "=&v"(r)
        : "v"(v), "v"(x), "n"(L), "n"(L + 1), "n"(L + 2), "n"(L + 3));
    return r;
}
// sum over k of (lane L + k of 16 of v) x[k]
template <int L>
__device__ inline float dot_lanes(float v, const float (&x)[H]) {
    float r;
    asm("s_nop 1\n\t"
        "v_mul_f32_dpp %0, %1, %2 row_newbcast:%4 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %3 row_newbcast:%5 row_mask:0xf bank_mask:0xf"
        : "=&v"(r)
        : "v"(v), "v"(x[0]), "v"(x[1]), "n"(L), "n"(L + 1));
    return r;
}

// What one of the asm blocks above wrote, before lanes exchange it: the exchange may read a
// register two wait states after a vector instruction wrote it, and the compiler counts
// them for its own instructions only.
__device__ inline void settle(float &x, float &y) { asm("s_nop 1" : "+v"(x), "+v"(y)); }

// Lanes add up pairs of registers so that half of the lanes go on with x's sum and half,
// those with the bit BIT of their number set, with y's.  The other lane of a pair is the
// one across BIT, for 4 across 7 and for 2 across 3 (a reversal is one instruction):
// taken in the order 32, 16, 8, 4, 2, 1 it has every earlier bit in common.
template <int BIT>
__device__ inline float halve(float x, float y) {
    if constexpr (BIT == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y),
                                                        false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else if constexpr (BIT == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y),
                                                        false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        // row_ror:8, row_half_mirror, quad_perm [3,2,1,0], quad_perm [1,0,3,2]
        constexpr int kCtrl = BIT == 8 ? 0x128 : BIT == 4 ? 0x141 : BIT == 2 ? 0x1b : 0xb1;
        const bool up = (threadIdx.x & BIT) != 0;
        const float keep = up ? y : x, give = up ? x : y;
        return keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(give), kCtrl,
                                                                 0xf, 0xf, false));
    }
}

// What the halves of a wave add to a token and channel.  Tokens come in pairs, either
// way: `first` holds the one that came first, with the second each half of the lanes ends
// with a token's sum, the even one's the lower, which lie side by side in LDS.  ASM: an asm
// block wrote the values.
template <int t, bool DOWN, bool ASM>
__device__ inline void put_pair(float *tile, int lane, bool more, float &first, float v) {
    if constexpr ((t % 2 == 1) == DOWN) {
        first = v;
    } else {
        if (ASM) settle(first, v);
        const float sum = DOWN ? halve<32>(v, first) : halve<32>(first, v);
        float *at = tile + (t & ~1) * kChans + lane;
        *at = more ? *at + sum : sum;
    }
}

// OUT: outputs (and saved states), from a.slot's or the caller's start; else the end
// state from zero and the sum of the steps, into a.slot and a.sums.
template <typename T, int W, bool MANY, bool OUT>
__global__ __launch_bounds__(kLanes * W) void selscan_kernel(Selscan a) {
    using G = Geo<W>;
    constexpr int EL = G::kEl, ROW = G::kRow, TOK = G::kTok;
    constexpr int RND = MANY ? kSelscanMaxStates / ROW : 1;
    __shared__ float2 sd[kTile][kChans];
    __shared__ Vecs vecs[RND][2 * W];
    __shared__ float yp[OUT ? W : 1][kTile][kChans];
    __shared__ float carry[MANY ? kSelscanMaxStates : 1][kChans];
    const int tid = threadIdx.x, lane = tid & 63, ch = lane & 31, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int st = tid / TOK, se = tid % TOK * EL, si = tid % TOK;  // staging
    const Place p = place_of(a, OUT ? a.segs : a.segs - 1);
    const int len = length_of(a, p.b), rounds = (a.N + ROW - 1) / ROW;
    const int begin = p.seg * a.seg_len, end = min(a.T, begin + a.seg_len);
    const int m = min(EL, max(0, p.live - se));
    const int64_t sbase = ((int64_t)p.b * a.N) * a.n + p.c0 + ch;  // state [b][0][c]
    const bool on = ch < p.live;
    const float *first = OUT && a.segs > 1
                             ? a.slot + (int64_t)p.seg * a.B * a.N * a.n
                             : OUT ? a.state_in : nullptr;
    float h[H], a2[H];
    auto state = [&](int r, int k) { return r * ROW + (2 * w + half) * H + k; };
    auto load_round = [&](int r) {
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const int i = state(r, k);
            const bool in = on && i < a.N;
            a2[k] = in ? rate(a.a[(int64_t)i * a.n + p.c0 + ch]) : 0.f;
            h[k] = in && first ? first[sbase + (int64_t)i * a.n] : 0.f;
        }
    };
    if (MANY) {
        for (int r = 0; r < rounds; ++r) {
            load_round(r);
#pragma unroll
            for (int k = 0; k < H; ++k) carry[state(r, k)][ch] = h[k];
        }
    } else {
        load_round(0);
    }
    float bias[EL], skip[EL], sum[EL];
#pragma unroll
    for (int j = 0; j < EL; ++j) {
        bias[j] = a.dt_bias && j < m ? a.dt_bias[p.c0 + se + j] : 0.f;
        skip[j] = a.skip && j < m ? a.skip[p.c0 + se + j] : 0.f;
        sum[j] = 0.f;
    }
    const int t1 = begin + st;
    const Walk<T> wu = walk_rows<T>(a.u, t1, p, se), wd = walk_rows<T>(a.dt, t1, p, se),
                  wz = walk_rows<T>(a.z, t1, p, se),
                  wy = walk_rows<T>(SelscanRows{a.y, a.y_st, a.y_sb}, t1, p, se),
                  wb = walk_vec<T>(a.b, t1, p, 0), wc = walk_vec<T>(a.c, t1, p, 0);
    Raw<T, EL> ru, rd, rz;
    T rb[RND], rc[RND];
    const int stop = min(end, len);
    // not converted yet: that would wait for the loads
    auto fetch = [&](int t0) {
        if (t0 + st >= stop) return;
        fetch_run(ru, wu.tile(t0 - begin), p, m);
        fetch_run(rd, wd.tile(t0 - begin), p, m);
        if (OUT && a.z.p) fetch_run(rz, wz.tile(t0 - begin), p, m);
#pragma unroll
        for (int r = 0; r < RND; ++r) {
            const int i = min(r * ROW + si, a.N - 1);
            rb[r] = wb.tile(t0 - begin)[i];
            if (OUT) rc[r] = wc.tile(t0 - begin)[i];
        }
    };
    // Outputs are stored once the next tile's loads are there: memory accesses end in
    // order, and those loads would be waited for together with a store before them.
    float out[EL] = {};
    auto write_out = [&](int t0) {
        if (t0 + st < end) put_run(wy.tile(t0 - begin), p, m, out);
    };
    if (begin < stop) fetch(begin);
    for (int t0 = begin; t0 < stop; t0 += kTile) {
        float u[EL], z[EL], d[EL];
        const bool in = t0 + st < stop;
        ru.get(u);
        rd.get(d);
        if (OUT && a.z.p) rz.get(z);
        steps<EL>(a.softplus, d, bias);
#pragma unroll
        for (int j = 0; j < EL; ++j) {
            d[j] = in && j < m ? d[j] : 0.f;
            sd[st][se + j] = make_float2(d[j], in ? d[j] * u[j] : 0.f);
            sum[j] += d[j];
        }
#pragma unroll
        for (int r = 0; r < RND; ++r) {
            if (si < ROW) {
                float *v = &vecs[r][si / H][0][0] + st * kSlots + si % H;
                const bool there = in && r * ROW + si < a.N;
                v[0] = there ? (float)rb[r] : 0.f;
                if (OUT) v[H] = there ? (float)rc[r] : 0.f;
            }
        }
        if (OUT && t0 > begin) write_out(t0 - kTile);
        if (t0 + kTile < stop) fetch(t0 + kTile);
        __syncthreads();
        for (int r = 0; r < (MANY ? rounds : 1); ++r) {
            if (MANY) {
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    const int i = state(r, k);
                    a2[k] = on && i < a.N ? rate(a.a[(int64_t)i * a.n + p.c0 + ch]) : 0.f;
                    h[k] = carry[i][ch];
                }
            }
            if (OUT && a.saved) {
                float *s = a.saved + (int64_t)(t0 / kTile) * a.B * a.N * a.n + sbase;
#pragma unroll
                for (int k = 0; k < H; ++k)
                    if (on && state(r, k) < a.N) s[(int64_t)state(r, k) * a.n] = h[k];
            }
            float vr = 0.f, pair = 0.f;
            (void)pair;
            each<kTile>([&](auto tt) {
                constexpr int t = decltype(tt)::value, at = t * kSlots % 16;
                if constexpr (at == 0) vr = vecs[r][2 * w + half][t * kSlots / 16][lane & 15];
                const float2 v = sd[t][ch];
                each<H>([&](auto kk) {
                    constexpr int k = decltype(kk)::value;
                    const float e = __builtin_amdgcn_exp2f(v.x * a2[k]);
                    h[k] = __builtin_fmaf(e, h[k], v.y * lane_of16<at + k>(vr));
                });
                if constexpr (OUT) put_pair<t, false, true>(&yp[w][0][0], lane, MANY && r, pair, dot_lanes<at + H>(vr, h));
            });
            if (MANY) {
#pragma unroll
                for (int k = 0; k < H; ++k) carry[state(r, k)][ch] = h[k];
            }
        }
        __syncthreads();
        if (OUT) {
            float y[EL];
#pragma unroll
            for (int j = 0; j < EL; ++j) {
                y[j] = yp[0][st][se + j];
#pragma unroll
                for (int k = 1; k < W; ++k) y[j] += yp[k][st][se + j];
                y[j] = __builtin_fmaf(skip[j], u[j], y[j]);
            }
            if (a.z.p)
#pragma unroll
                for (int j = 0; j < EL; ++j) y[j] *= silu<sizeof(T) == 4>(z[j]);
#pragma unroll
            for (int j = 0; j < EL; ++j) y[j] = in ? y[j] : 0.f;
#pragma unroll
            for (int j = 0; j < EL; ++j) out[j] = y[j];
        }
    }
    if (OUT && begin < stop) write_out((stop - begin - 1) / kTile * kTile + begin);
    // rows past the sequence, from the first tile that the loop left out
    if (OUT) {
        const float none[EL] = {};
        const int from = begin < stop ? begin + (stop - begin + kTile - 1) / kTile * kTile : begin;
        for (int t = from; t + st < end; t += kTile) put_run(wy.tile(t - begin), p, m, none);
    }
    float *last = OUT ? (p.seg == a.segs - 1 ? a.state_out : nullptr)
                      : a.slot + (int64_t)p.seg * a.B * a.N * a.n;
    if (last)
        for (int r = 0; r < (MANY ? rounds : 1); ++r)
#pragma unroll
            for (int k = 0; k < H; ++k) {
                const int i = state(r, k);
                if (on && i < a.N)
                    last[sbase + (int64_t)i * a.n] = MANY ? carry[i][ch] : h[k];
            }
    if (!OUT) {  // the steps' sum: over the staging threads of a channel
        __syncthreads();
        float *s = &sd[0][0].x;
#pragma unroll
        for (int j = 0; j < EL; ++j) s[st * kChans + se + j] = sum[j];
        __syncthreads();
        if (w == 0 && half == 0 && on) {
            float t = 0.f;
            for (int k = 0; k < kTile; ++k) t += s[k * kChans + ch];
            a.sums[((int64_t)p.seg * a.B + p.b) * a.n + p.c0 + ch] = t;
        }
    }
}

// Joins the segments: slot s, a segment's end state from zero, becomes the state that
// enters it (reverse: the gradient of the state that leaves it).
__global__ __launch_bounds__(256) void selscan_join_kernel(Selscan a, const float *from,
                                                           bool reverse) {
    // fewer than 2^32 states in all
    const uint32_t e = blockIdx.x * 256 + threadIdx.x;
    const int64_t size = (int64_t)a.B * a.N * a.n;
    if (e >= size) return;
    const uint32_t row = e / (uint32_t)a.n, c = e - row * a.n, b = row / a.N, i = row - b * a.N;
    const float a2 = rate(a.a[(int64_t)i * a.n + c]);
    float h = from ? from[e] : 0.f;
    constexpr int AHEAD = 8;  // segments on their way: one after the other they cost 12 us
    for (int k0 = 0; k0 < a.segs; k0 += AHEAD) {
        float own[AHEAD], d[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = min(k0 + j, a.segs - 2), s = reverse ? a.segs - 1 - k : k;
            own[j] = a.slot[s * size + e];
            d[j] = a.sums[((int64_t)s * a.B + b) * a.n + c];
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = k0 + j;
            if (k >= a.segs) break;
            a.slot[(reverse ? a.segs - 1 - k : k) * size + e] = h;
            h = __builtin_fmaf(__builtin_amdgcn_exp2f(d[j] * a2), h, own[j]);
        }
    }
}

// ---- backward ------------------------------------------------------------------------

template <typename T, int W, bool MANY>
__global__ __launch_bounds__(kLanes * W, 2) void selscan_bwd_kernel(SelscanBwd q) {
    using G = Geo<W>;
    const Selscan &a = q.a;
    constexpr int EL = G::kEl, ROW = G::kRow, TOK = G::kTok;
    constexpr int RND = MANY ? kSelscanMaxStates / ROW : 1;
    __shared__ float2 sd[kTile][kChans];  // step, step times u
    __shared__ float sg[kTile][kChans];
    __shared__ Vecs vecs[RND][2 * W];
    __shared__ float yp[W][kTile][kChans], up[W][kTile][kChans], dp[W][kTile][kChans];
    __shared__ float carry[MANY ? kSelscanMaxStates : 1][kChans];
    __shared__ float asum[MANY ? kSelscanMaxStates : 1][kChans];
    const int tid = threadIdx.x, lane = tid & 63, ch = lane & 31, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int st = tid / TOK, se = tid % TOK * EL, si = tid % TOK;
    const Place p = place_of(a, a.segs);
    const int len = length_of(a, p.b), rounds = (a.N + ROW - 1) / ROW;
    const int begin = p.seg * a.seg_len, end = min(a.T, begin + a.seg_len);
    const int m = min(EL, max(0, p.live - se));
    const int64_t sbase = ((int64_t)p.b * a.N) * a.n + p.c0 + ch;
    const bool on = ch < p.live;
    const float *first = a.segs > 1 ? a.slot + (int64_t)p.seg * a.B * a.N * a.n
                                    : q.grad_state_out;
    float g[H], a2[H], acc[H];
    auto state = [&](int r, int k) { return r * ROW + (2 * w + half) * H + k; };
    for (int r = 0; r < (MANY ? rounds : 1); ++r)
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const int i = state(r, k);
            const bool in = on && i < a.N;
            a2[k] = in ? rate(a.a[(int64_t)i * a.n + p.c0 + ch]) : 0.f;
            g[k] = in && first ? first[sbase + (int64_t)i * a.n] : 0.f;
            acc[k] = 0.f;
            if (MANY) carry[i][ch] = g[k], asum[i][ch] = 0.f;
        }
    float gskip[EL] = {}, gbias[EL] = {}, bias[EL] = {}, skip[EL] = {};
    if (a.dt_bias) load_run(a.dt_bias + p.c0 + se, m, bias);
    if (a.skip) load_run(a.skip + p.c0 + se, m, skip);
    float hs[H];  // the states before a tile, on their way while the one after it is run
    auto fetch_states = [&](int t0, int r) {
        const float *s = q.saved + (int64_t)(t0 / kTile) * a.B * a.N * a.n + sbase - (on ? 0 : ch);
#pragma unroll
        for (int k = 0; k < H; ++k) hs[k] = s[(int64_t)min(state(r, k), a.N - 1) * a.n];
    };
    const int t1 = begin + st;
    const Walk<T> wu = walk_rows<T>(a.u, t1, p, se), wd = walk_rows<T>(a.dt, t1, p, se),
                  wz = walk_rows<T>(a.z, t1, p, se),
                  wg = walk_rows<T>(SelscanRows{q.gy, a.y_st, a.y_sb}, t1, p, se),
                  wdu = walk_rows<T>(q.du, t1, p, se), wdd = walk_rows<T>(q.ddt, t1, p, se),
                  wdz = walk_rows<T>(q.dz, t1, p, se), wb = walk_vec<T>(a.b, t1, p, 0),
                  wc = walk_vec<T>(a.c, t1, p, 0);
    Raw<T, EL> ru, rd, rz, rg;
    T rb[RND], rc[RND];
    const int stop = min(end, len);
    auto fetch = [&](int t0) {
        if (t0 + st >= stop) return;
        fetch_run(ru, wu.tile(t0 - begin), p, m);
        fetch_run(rd, wd.tile(t0 - begin), p, m);
        fetch_run(rg, wg.tile(t0 - begin), p, m);
        if (a.z.p) fetch_run(rz, wz.tile(t0 - begin), p, m);
#pragma unroll
        for (int r = 0; r < RND; ++r) {
            const int i = min(r * ROW + si, a.N - 1);
            rb[r] = wb.tile(t0 - begin)[i];
            rc[r] = wc.tile(t0 - begin)[i];
        }
    };
    const float none[EL] = {};
    // rows past the sequence
    for (int t = max(begin, stop); t + st < end; t += kTile) {
        put_run(wdu.tile(t - begin), p, m, none);
        put_run(wdd.tile(t - begin), p, m, none);
        if (a.z.p) put_run(wdz.tile(t - begin), p, m, none);
    }
    // sums over this workgroup's channels: a lane's token and integrator
    const int per = a.tiles / a.groups;
    const int vt = (lane >> 2 & 1) + (lane & 2) + (lane & 1) * 4;
    const int vi = (2 * w + half) * H + (lane >> 3 & 1);
    const int64_t vstep = (int64_t)a.B * a.groups * a.N;
    const Walk<float> wv{q.vec + (((int64_t)(lane >> 4 & 1) * per + p.tile % per) * a.T + begin + vt) *
                                     vstep +
                             (p.b * a.groups + p.g) * a.N + vi,
                         vstep};
    const int tiles = begin < stop ? (stop - begin + kTile - 1) / kTile : 0;
    if (tiles > 0) {
        fetch(begin + (tiles - 1) * kTile);
        if (!MANY) fetch_states(begin + (tiles - 1) * kTile, 0);
    }
    for (int x = tiles - 1; x >= 0; --x) {
        const int t0 = begin + x * kTile;
        const bool in = t0 + st < stop;
        float u[EL], slope[EL], zs[EL] = {};  // zs: gradient of the gate's input over y
        {
            float d[EL], gy[EL];
            ru.get(u);
            rd.get(d);
            rg.get(gy);
            if (a.z.p) rz.get(zs);
#pragma unroll
            for (int j = 0; j < EL; ++j) {
                slope[j] = 1.f;
                d[j] += bias[j];
            }
            if (a.softplus)
#pragma unroll
                for (int j = 0; j < EL; ++j) softplus(d[j], d[j], slope[j]);
            float gi[EL];
#pragma unroll
            for (int j = 0; j < EL; ++j) gi[j] = gy[j];
            if (a.z.p)
#pragma unroll
                for (int j = 0; j < EL; ++j) {
                    float act;
                    silu_slope<sizeof(T) == 4>(zs[j], act, zs[j]);
                    gi[j] *= act;
                    zs[j] *= gy[j];
                }
#pragma unroll
            for (int j = 0; j < EL; ++j) {
                d[j] = in && j < m ? d[j] : 0.f;
                u[j] = in ? u[j] : 0.f;
                sd[st][se + j] = make_float2(d[j], d[j] * u[j]);
                sg[st][se + j] = in ? gi[j] : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < RND; ++r) {
            if (si < ROW) {
                float *v = &vecs[r][si / H][0][0] + st * kSlots + si % H;
                const bool there = in && r * ROW + si < a.N;
                v[0] = there ? (float)rb[r] : 0.f;
                v[H] = there ? (float)rc[r] : 0.f;
            }
        }
        if (x > 0) fetch(t0 - kTile);
        __syncthreads();
        for (int r = 0; r < (MANY ? rounds : 1); ++r) {
            const int i0 = state(r, 0);
            float h0[H], h[kTile][H], e[kTile][H];
            if (MANY) fetch_states(t0, r);
#pragma unroll
            for (int k = 0; k < H; ++k) {
                h0[k] = hs[k];
                if (MANY) {
                    a2[k] = on && i0 + k < a.N
                                ? rate(a.a[(int64_t)(i0 + k) * a.n + p.c0 + ch])
                                : 0.f;
                    g[k] = carry[i0 + k][ch];
                    acc[k] = asum[i0 + k][ch];
                }
            }
            if (!MANY && x > 0) fetch_states(t0 - kTile, 0);
            // the tile's values of this lane, for both directions
            float vrs[kVecRows], gvs[kTile], pair[2];
            float2 dus[kTile];
#pragma unroll
            for (int k = 0; k < kVecRows; ++k) vrs[k] = vecs[r][2 * w + half][k][lane & 15];
#pragma unroll
            for (int t = 0; t < kTile; ++t) dus[t] = sd[t][ch];
#pragma unroll
            for (int t = kTile - 1; t >= 0; --t) gvs[t] = sg[t][ch];
            each<kTile>([&](auto tt) {
                constexpr int t = decltype(tt)::value, at = t * kSlots % 16;
                const float vr = vrs[t * kSlots / 16], dv = dus[t].x, uv = dus[t].y;
                each<H>([&](auto kk) {
                    constexpr int k = decltype(kk)::value;
                    e[t][k] = __builtin_amdgcn_exp2f(dv * a2[k]);
                    h[t][k] = __builtin_fmaf(e[t][k], t ? h[t ? t - 1 : 0][k] : h0[k],
                                             uv * lane_of16<at + k>(vr));
                });
                // only the gate's gradient wants it: without a condition the tokens are one
                // stretch of code
                put_pair<t, false, true>(&yp[w][0][0], lane, MANY && r, pair[0], dot_lanes<at + H>(vr, h[t]));
            });
            // a's gradient: the tile's sum, then the tiles', a chain of T / 16 + 16 additions
            // (token by token 8192 equal ones were off by 2000 units, in the same time)
            float part[3], da[H] = {};
            each<kTile>([&](auto tt) {
                constexpr int t = kTile - 1 - decltype(tt)::value, at = t * kSlots % 16;
                const float vr = vrs[t * kSlots / 16], dv = dus[t].x, uv = dus[t].y, gv = gvs[t];
                float gd = 0.f, vb[H], vc[H];
                const float gin = fma_dot_lanes<at>(g, vr, gv);
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    vc[k] = gv * h[t][k];
                    vb[k] = g[k] * uv;
                    g[k] *= e[t][k];
                    const float x_ = g[k] * (t ? h[t ? t - 1 : 0][k] : h0[k]);
                    da[k] = __builtin_fmaf(x_, dv, da[k]);
                    gd = __builtin_fmaf(x_, a2[k], gd);
                }
                put_pair<t, true, true>(&up[w][0][0], lane, MANY && r, pair[0], gin);
                put_pair<t, true, false>(&dp[w][0][0], lane, MANY && r, pair[1], gd);
                // The sums over lanes.  Bits of the lane that a sum ends in: 16 b or c, 8
                // the integrator's, then the token's from the low one on.  Tokens are joined
                // in pairs, fours and eights.
                float v = halve<8>(halve<16>(vb[0], vc[0]), halve<16>(vb[1], vc[1]));
                each<3>([&](auto ll) {
                    constexpr int l = decltype(ll)::value;
                    if constexpr ((t & ((1 << l) - 1)) == 0) {
                        if constexpr (t >> l & 1) part[l] = v;
                        else v = halve<(4 >> l)>(v, part[l]);
                    }
                });
                if constexpr (t % 8 == 0) {
                    if (t0 + t + vt < stop && vi + r * ROW < a.N)
                        wv.tile(t0 + t - begin)[r * ROW] = v;
                }
            });
#pragma unroll
            for (int k = 0; k < H; ++k) acc[k] += da[k];
            if (MANY) {
#pragma unroll
                for (int k = 0; k < H; ++k) carry[i0 + k][ch] = g[k], asum[i0 + k][ch] = acc[k];
            }
        }
        __syncthreads();
        float gu[EL], gdt[EL];
#pragma unroll
        for (int j = 0; j < EL; ++j) {
            float y = a.z.p ? yp[0][st][se + j] : 0.f, gin = up[0][st][se + j],
                  gd = dp[0][st][se + j];
#pragma unroll
            for (int k = 1; k < W; ++k) {
                if (a.z.p) y += yp[k][st][se + j];
                gin += up[k][st][se + j];
                gd += dp[k][st][se + j];
            }
            const float d = sd[st][se + j].x, gi = sg[st][se + j];
            gu[j] = __builtin_fmaf(gin, d, gi * skip[j]);
            gdt[j] = in ? __builtin_fmaf(gin, u[j], gd * kLn2) * slope[j] : 0.f;
            zs[j] *= __builtin_fmaf(skip[j], u[j], y);
            gskip[j] = __builtin_fmaf(gi, u[j], gskip[j]);
            gbias[j] += gdt[j];
        }
        if (in) {
            put_run(wdu.tile(t0 - begin), p, m, gu);
            put_run(wdd.tile(t0 - begin), p, m, gdt);
            if (a.z.p) put_run(wdz.tile(t0 - begin), p, m, zs);
        }
    }
    // the gradient of the state before the segment, and the sums over its tokens
    float *last = p.seg == 0 ? q.grad_state_in : nullptr;
    float *rows = q.part + ((int64_t)p.b * a.segs + p.seg) * (a.N + 2) * a.n + p.c0 + ch;
    for (int r = 0; r < (MANY ? rounds : 1); ++r)
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const int i = state(r, k);
            if (on && i < a.N) {
                if (last) last[sbase + (int64_t)i * a.n] = MANY ? carry[i][ch] : g[k];
                rows[(int64_t)i * a.n] = MANY ? asum[i][ch] : acc[k];
            }
        }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EL; ++j) sd[st][se + j] = make_float2(gskip[j], gbias[j]);
    __syncthreads();
    if (w == 0 && half == 0 && on) {
        float s0 = 0.f, s1 = 0.f;
        for (int k = 0; k < kTile; ++k) s0 += sd[k][ch].x, s1 += sd[k][ch].y;
        rows[(int64_t)a.N * a.n] = s0;
        rows[(int64_t)(a.N + 1) * a.n] = s1;
    }
}

// The gradient that a segment passes on from its own tokens, and the sum of its steps:
// segments 1 .. segs - 1.
template <typename T, int W, bool MANY>
__global__ __launch_bounds__(kLanes * W) void selscan_back_kernel(SelscanBwd q) {
    using G = Geo<W>;
    const Selscan &a = q.a;
    constexpr int EL = G::kEl, ROW = G::kRow, TOK = G::kTok;
    constexpr int RND = MANY ? kSelscanMaxStates / ROW : 1;
    __shared__ float2 sd[kTile][kChans];
    __shared__ Vecs vecs[RND][2 * W];
    __shared__ float carry[MANY ? kSelscanMaxStates : 1][kChans];
    const int tid = threadIdx.x, lane = tid & 63, ch = lane & 31, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int st = tid / TOK, se = tid % TOK * EL, si = tid % TOK;
    Place p = place_of(a, a.segs - 1);
    p.seg += 1;
    const int len = length_of(a, p.b), rounds = (a.N + ROW - 1) / ROW;
    const int begin = p.seg * a.seg_len, end = min(a.T, begin + a.seg_len);
    const int m = min(EL, max(0, p.live - se));
    const int64_t sbase = ((int64_t)p.b * a.N) * a.n + p.c0 + ch;
    const bool on = ch < p.live;
    float g[H], a2[H];
    auto state = [&](int r, int k) { return r * ROW + (2 * w + half) * H + k; };
    auto rates = [&](int r) {
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const int i = state(r, k);
            a2[k] = on && i < a.N ? rate(a.a[(int64_t)i * a.n + p.c0 + ch]) : 0.f;
        }
    };
    rates(0);
#pragma unroll
    for (int k = 0; k < H; ++k) g[k] = 0.f;
    // by the lanes that read them: a segment past the sequence's end has no barrier between
    if (MANY)
        for (int r = 0; r < rounds; ++r)
#pragma unroll
            for (int k = 0; k < H; ++k) carry[state(r, k)][ch] = 0.f;
    float bias[EL], sum[EL];
#pragma unroll
    for (int j = 0; j < EL; ++j) {
        bias[j] = a.dt_bias && j < m ? a.dt_bias[p.c0 + se + j] : 0.f;
        sum[j] = 0.f;
    }
    const int t1 = begin + st;
    const Walk<T> wd = walk_rows<T>(a.dt, t1, p, se), wz = walk_rows<T>(a.z, t1, p, se),
                  wg = walk_rows<T>(SelscanRows{q.gy, a.y_st, a.y_sb}, t1, p, se),
                  wc = walk_vec<T>(a.c, t1, p, 0);
    Raw<T, EL> rd, rz, rg;
    T rc[RND];
    const int stop = min(end, len);
    auto fetch = [&](int t0) {
        if (t0 + st >= stop) return;
        fetch_run(rd, wd.tile(t0 - begin), p, m);
        fetch_run(rg, wg.tile(t0 - begin), p, m);
        if (a.z.p) fetch_run(rz, wz.tile(t0 - begin), p, m);
#pragma unroll
        for (int r = 0; r < RND; ++r) rc[r] = wc.tile(t0 - begin)[min(r * ROW + si, a.N - 1)];
    };
    const int tiles = begin < stop ? (stop - begin + kTile - 1) / kTile : 0;
    if (tiles > 0) fetch(begin + (tiles - 1) * kTile);
    for (int x = tiles - 1; x >= 0; --x) {
        const int t0 = begin + x * kTile;
        const bool in = t0 + st < stop;
        float z[EL], d[EL], gy[EL];
        rd.get(d);
        rg.get(gy);
        if (a.z.p) rz.get(z);
        __syncthreads();  // the tile before has been read
        steps<EL>(a.softplus, d, bias);
        if (a.z.p)
#pragma unroll
            for (int j = 0; j < EL; ++j) gy[j] *= silu<sizeof(T) == 4>(z[j]);
#pragma unroll
        for (int j = 0; j < EL; ++j) {
            d[j] = in && j < m ? d[j] : 0.f;
            sd[st][se + j] = make_float2(d[j], in ? gy[j] : 0.f);
            sum[j] += d[j];
        }
#pragma unroll
        for (int r = 0; r < RND; ++r)
            if (si < ROW)
                (&vecs[r][si / H][0][0])[st * kSlots + H + si % H] =
                    in && r * ROW + si < a.N ? (float)rc[r] : 0.f;
        if (x > 0) fetch(t0 - kTile);
        __syncthreads();
        for (int r = 0; r < (MANY ? rounds : 1); ++r) {
            const int i0 = state(r, 0);
            if (MANY) {
                rates(r);
#pragma unroll
                for (int k = 0; k < H; ++k) g[k] = carry[i0 + k][ch];
            }
            float vr = 0.f;
            each<kTile>([&](auto tt) {
                constexpr int t = kTile - 1 - decltype(tt)::value, at = t * kSlots % 16;
                if constexpr (at + kSlots == 16) vr = vecs[r][2 * w + half][t * kSlots / 16][lane & 15];
                const float2 v = sd[t][ch];
                each<H>([&](auto kk) {
                    constexpr int k = decltype(kk)::value;
                    fma_lane<at + H + k>(g[k], vr, v.y);
                    g[k] *= __builtin_amdgcn_exp2f(v.x * a2[k]);
                });
            });
            if (MANY) {
#pragma unroll
                for (int k = 0; k < H; ++k) carry[i0 + k][ch] = g[k];
            }
        }
    }
    for (int r = 0; r < (MANY ? rounds : 1); ++r)
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const int i = state(r, k);
            if (on && i < a.N)
                a.slot[(int64_t)p.seg * a.B * a.N * a.n + sbase + (int64_t)i * a.n] =
                    MANY ? carry[i][ch] : g[k];
        }
    __syncthreads();
    float *s = &sd[0][0].x;
#pragma unroll
    for (int j = 0; j < EL; ++j) s[st * kChans + se + j] = sum[j];
    __syncthreads();
    if (w == 0 && half == 0 && on) {
        float t = 0.f;
        for (int k = 0; k < kTile; ++k) t += s[k * kChans + ch];
        a.sums[((int64_t)p.seg * a.B + p.b) * a.n + p.c0 + ch] = t;
    }
}

// `count` values `step` apart added in order, 16 on their way at a time
__device__ inline float ordered_sum(const float *p, int64_t step, int count) {
    float s = 0.f;
    for (int k0 = 0; k0 < count; k0 += 16) {
        float x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = k0 + j < count ? p[(k0 + j) * step] : 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) s += x[j];
    }
    return s;
}

// Gradients of b and c: the channel tiles' sums, in order; tokens past a sequence 0.
template <typename T>
__global__ __launch_bounds__(256) void selscan_vec_kernel(SelscanBwd q) {
    const Selscan &a = q.a;
    const int64_t per = (int64_t)a.T * a.B * a.groups * a.N;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= per) return;
    const int which = blockIdx.y, tiles = a.tiles / a.groups;
    const int gi = (int)(e % (a.groups * a.N)), i = gi % a.N, g = gi / a.N;
    const int64_t tb = e / (a.groups * a.N);
    const int b = (int)(tb % a.B), t = (int)(tb / a.B);
    float s = 0.f;
    if (t < length_of(a, b)) {
        s = ordered_sum(q.vec + which * tiles * per + e, per, tiles);
    }
    const SelscanVec &v = which ? q.dc : q.db;
    static_cast<T *>(const_cast<void *>(v.p))[t * v.st + b * v.sb + g * v.sg + i] = (T)s;
}

// Gradients of a, skip and dt_bias: the sequences' and segments' sums, in order.
__global__ __launch_bounds__(256) void selscan_rows_kernel(SelscanBwd q, int rows) {
    const Selscan &a = q.a;
    const int64_t size = (int64_t)(a.N + 2) * a.n;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= size) return;
    const int i = (int)(e / a.n);
    float *out = i < a.N ? q.grad_a : i == a.N ? q.grad_skip : q.grad_dt_bias;
    if (!out) return;
    const float s = ordered_sum(q.part + e, size, rows);
    out[i < a.N ? e : e % a.n] = s;
}

// ---- one token -----------------------------------------------------------------------
// Bound by HBM, by the states read and written once.  A thread takes a channel of a
// request, eight of its integrators on their way at a time (64 requests of 4096 channels
// of 16: 9.0 us, 3.8 TB/s; four channels a thread leave too few waves, 16.4).
template <typename T>
__global__ __launch_bounds__(256) void selscan_step_kernel(Selscan a, const int32_t *slots,
                                                           int n_slots) {
    const int per = (a.n + 255) / 256, b = blockIdx.x / per;
    const int c = (blockIdx.x - b * per) * 256 + threadIdx.x;
    if (c >= a.n) return;
    T *y = static_cast<T *>(a.y) + b * a.y_sb + c;
    const int slot = slots ? slots[b] : b;
    if (slot < 0 || slot >= n_slots) {
        *y = (T)0.f;
        return;
    }
    const float u = (float)static_cast<const T *>(a.u.p)[b * a.u.sb + c];
    float d = (float)static_cast<const T *>(a.dt.p)[b * a.dt.sb + c];
    const float z = a.z.p ? (float)static_cast<const T *>(a.z.p)[b * a.z.sb + c] : 0.f;
    const float skip = a.skip ? a.skip[c] : 0.f, bias = a.dt_bias ? a.dt_bias[c] : 0.f;
    const int g = a.groups == 1 ? 0 : c / (a.n / a.groups);
    const T *pb = static_cast<const T *>(a.b.p) + b * a.b.sb + g * a.b.sg;
    const T *pc = static_cast<const T *>(a.c.p) + b * a.c.sb + g * a.c.sg;
    const float *in = a.state_in + (int64_t)slot * a.N * a.n + c;
    float *to = a.state_out + (int64_t)slot * a.N * a.n + c;
    constexpr int AHEAD = 8;
    float du = 0.f, out = 0.f;
    for (int i0 = 0; i0 < a.N; i0 += AHEAD) {
        float h[AHEAD], r[AHEAD];
        T bv[AHEAD], cv[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = min(i0 + k, a.N - 1);
            h[k] = in[(int64_t)i * a.n];
            r[k] = a.a[(int64_t)i * a.n + c];
            bv[k] = pb[i];
            cv[k] = pc[i];
        }
        if (i0 == 0) {  // behind the first loads
            float slope;
            d += bias;
            if (a.softplus) softplus(d, d, slope);
            du = d * u;
            d *= kLog2e;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k >= a.N) break;
            h[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * r[k]), h[k], du * (float)bv[k]);
            out = __builtin_fmaf((float)cv[k], h[k], out);
            to[(int64_t)(i0 + k) * a.n] = h[k];
        }
    }
    out = __builtin_fmaf(skip, u, out);
    if (a.z.p) out *= silu<sizeof(T) == 4>(z);
    *y = (T)out;
}

template <typename T, int W, bool MANY>
hipError_t run_fwd(const Selscan &a, hipStream_t s) {
    const int units = a.tiles * a.B, threads = Geo<W>::kThreads;
    if (a.segs > 1) {
        selscan_kernel<T, W, MANY, false><<<units * (a.segs - 1), threads, 0, s>>>(a);
        const int64_t size = (int64_t)a.B * a.N * a.n;
        selscan_join_kernel<<<(unsigned)((size + 255) / 256), 256, 0, s>>>(a, a.state_in, false);
    }
    selscan_kernel<T, W, MANY, true><<<units * a.segs, threads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int W, bool MANY>
hipError_t run_bwd(const SelscanBwd &q, hipStream_t s) {
    const Selscan &a = q.a;
    const int units = a.tiles * a.B, threads = Geo<W>::kThreads;
    if (units > 0 && a.segs > 1) {
        selscan_back_kernel<T, W, MANY><<<units * (a.segs - 1), threads, 0, s>>>(q);
        const int64_t size = (int64_t)a.B * a.N * a.n;
        selscan_join_kernel<<<(unsigned)((size + 255) / 256), 256, 0, s>>>(a, q.grad_state_out,
                                                                          true);
    }
    if (units > 0) selscan_bwd_kernel<T, W, MANY><<<units * a.segs, threads, 0, s>>>(q);
    const int64_t per = (int64_t)a.T * a.B * a.groups * a.N;
    if (per > 0)
        selscan_vec_kernel<T><<<dim3((unsigned)((per + 255) / 256), 2), 256, 0, s>>>(q);
    if (q.grad_a || q.grad_skip || q.grad_dt_bias)
        selscan_rows_kernel<<<(unsigned)(((int64_t)(a.N + 2) * a.n + 255) / 256), 256, 0, s>>>(
            q, a.B * a.segs);
    return hipGetLastError();
}

// Two waves for up to 8 integrators: 512 x 64 tokens of 1024 channels of 8, bf16, there and
// back 450 us, in four waves half of whose integrators are none 654 (512 x 16: 222, 209).
template <typename T>
hipError_t by_states(const Selscan &a, hipStream_t s) {
    if (a.N <= 8) return run_fwd<T, 2, false>(a, s);
    if (a.N <= 16) return run_fwd<T, 4, false>(a, s);
    return run_fwd<T, 4, true>(a, s);
}
template <typename T>
hipError_t by_states(const SelscanBwd &q, hipStream_t s) {
    if (q.a.N <= 8) return run_bwd<T, 2, false>(q, s);
    if (q.a.N <= 16) return run_bwd<T, 4, false>(q, s);
    return run_bwd<T, 4, true>(q, s);
}

template <typename T>
void run_step(const Selscan &a, const int32_t *slots, int n_slots, hipStream_t s) {
    selscan_step_kernel<T><<<a.B * ((a.n + 255) / 256), 256, 0, s>>>(a, slots, n_slots);
}

}  // namespace

int selscan_tiles(int n, int groups) {
    return groups * ((n / groups + kChans - 1) / kChans);
}

// Workgroups of 32 channels of a sequence, and of segments of it while they leave three
// eighths of the places (two to a compute unit) empty: the forward's eight to a unit, the
// backward's four.  1024 tokens, 16 integrators, bf16, there and back: 288 workgroups in
// segments 310 us, 384 uncut 375, as any from 257 to 512.
SelscanPlan selscan_plan(int T, int64_t units, bool backward) {
    SelscanPlan p{1, std::max(T, 1)};
    if (units < 1 || units > kPlanCus * 5 / 4) return p;
    const int tiles = (T + kTile - 1) / kTile, most = backward ? 4 : 8;
    const int segs = (int)std::min<int64_t>(most * kPlanCus / units, tiles / 4);
    if (segs < 2) return p;
    p.seg_len = (tiles + segs - 1) / segs * kTile;
    p.segs = (T + p.seg_len - 1) / p.seg_len;
    return p;
}

hipError_t launch_selscan(const Selscan &a, int dtype, hipStream_t s) {
    switch (dtype) {
        case SNN_F32: return by_states<float>(a, s);
        case SNN_F16: return by_states<half_t>(a, s);
        default: return by_states<bf16_t>(a, s);
    }
}

hipError_t launch_selscan_bwd(const SelscanBwd &q, int dtype, hipStream_t s) {
    switch (dtype) {
        case SNN_F32: return by_states<float>(q, s);
        case SNN_F16: return by_states<half_t>(q, s);
        default: return by_states<bf16_t>(q, s);
    }
}

hipError_t launch_selscan_step(const Selscan &a, const int32_t *slots, int n_slots, int dtype,
                               hipStream_t s) {
    switch (dtype) {
        case SNN_F32: run_step<float>(a, slots, n_slots, s); break;
        case SNN_F16: run_step<half_t>(a, slots, n_slots, s); break;
        default: run_step<bf16_t>(a, slots, n_slots, s); break;
    }
    return hipGetLastError();
}

}  // namespace snn
