// New tokens of a step: norm of every query and key head, rotation by position, the queries stored for the step and the keys and
// values written to the cache, bf16 or 4-bit, in one pass over the projections; and a 4-bit cache read back as a bf16 one.
//
//   y = x * w / sqrt(mean_c x_c^2 + eps);   (a, b) -> (a cos - b sin, a sin + b cos),  angle = position * inv_freq
//
// A warp takes a row's heads two (d = 128) or four (64) at a time, eight channels per lane, so that a head's sum is a few shuffles away;
// everything is read once and written once.  Few rows take latency: 8 rows 4.5 us.  Many are bound by no single thing: 8229 rows of 32 + 8 + 8 heads of
// 128, bf16, take 49 us (202 MB: 4.1 TB/s, 62 % of a copy's rate), in which 24 M warp instructions fill 48 % of the issue slots, at sixteen
// warps an SM that wait for their loads most.  32768 rows into the 4-bit cache and back take 248 us (883 MB: 3.6 TB/s): 210 for the write (137 M
// instructions, 59 % of the slots), 38 for the way back (31 M, 77 %: the index arithmetic, 64-bit divisions among it, is what a group's 41 bytes cost).
#include <math.h>
#include <string.h>

#include <type_traits>

#include "eta_attend.cuh"
#include "eta_kv4.cuh"

namespace eta {

struct TokensArgs {
    const void *q, *k, *v;
    const float *q_weight, *k_weight;
    const double* inv_freq;
    const int32_t* positions;
    const int64_t* slot_map;
    __nv_bfloat16 *q_out, *K, *V;
    unsigned char* pool;
    uint32_t* status;
    int64_t q_sr, q_sh, k_sr, k_sh, v_sr, v_sh;       // elements
    int64_t ks_b, ks_h, ks_t, vs_b, vs_h, vs_t;       // bf16 cache: elements; 4-bit: ks_* in bytes (page or sequence, head, block)
    int64_t limit;                                    // slots of the cache
    int rows, Hq, Hkv, per_page, b, q_parts, kv_parts, rotary, interleaved;
    FastDiv div_page, div_ctas;
    int ctas_row;          // CTAs of a row; 0: two rows to a CTA
    float k_scale, v_scale;
    // bit 0, 1: the keys', the values' scale leaves fp32 its range, and its product with a group's is exact (20 bits).  Of another scale everything is
    // worked out in fp64: 32768 rows take 682 us instead of 217 (bf16; 755 instead of 295 in fp32).
    int fast;
    float eps;
};

// eight consecutive channels
template <typename T>
struct Piece {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p, bool on) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
            w[k] = make_uint4(0, 0, 0, 0);
            if (on) w[k] = __ldcg(reinterpret_cast<const uint4*>(p) + k);
        }
    }
    // the piece of another lane
    __device__ __forceinline__ void exchange(int from) {
        uint32_t* u = reinterpret_cast<uint32_t*>(w);
#pragma unroll
        for (int k = 0; k < 2 * (int)sizeof(T); ++k) u[k] = __shfl_sync(0xffffffffu, u[k], from);
    }
    template <typename F>
    __device__ __forceinline__ void get(F (&x)[8]) const {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (sizeof(T) == 4) x[k] = (F)__uint_as_float(u[k]);
            else if constexpr (std::is_same<T, __half>::value) x[k] = (F)((k & 1) ? f16_hi(u[k / 2]) : f16_lo(u[k / 2]));
            else x[k] = (F)((k & 1) ? bf16_hi(u[k / 2]) : bf16_lo(u[k / 2]));
        }
    }
};

__device__ __forceinline__ uint4 pack_bf16(const float (&x)[8]) {
    uint4 o;
    uint32_t* u = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
        u[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return o;
}

// Sine and cosine of a row's pair.  The 64-bit angle is reduced by whole quarter turns with a two-part pi / 2 (Cody and Waite; the first difference
// is exact, so that what is left is as good as 64 bits however little that is): any 32-bit position keeps its angle, and next to a multiple of pi / 2
// the small one of the two is the sine of a small number, whose relative error F's rounding keeps small.  Rounding the angle itself to fp32
// moved a small factor by up to 2^-23 whatever its size.
__device__ __forceinline__ void sincos_of(float x, float* s, float* c) { sincosf(x, s, c); }
__device__ __forceinline__ void sincos_of(double x, double* s, double* c) { sincos(x, s, c); }
template <typename F>
__device__ __forceinline__ void turn_of(const TokensArgs& a, int64_t row, int pair, F& sn, F& cs) {
    const double x = (double)__ldcg(a.positions + row) * __ldcg(a.inv_freq + pair), n = rint(x * 0.6366197723675814);
    const int quarters = (int)__double2ll_rn(n);
    F s, c;
    sincos_of((F)fma(-n, 6.123233995736766e-17, fma(-n, 1.5707963267948966, x)), &s, &c);
    sn = (quarters & 1) ? c : s;
    cs = (quarters & 1) ? -s : c;
    if (quarters & 2) { sn = -sn; cs = -cs; }
}

// What a lane's eight channels are multiplied with, norm weight and rotation in one: y = (x C + x_partner S) r, where x_partner are the pairs'
// other channels as they came, C = w cos, S = -+ w_partner sin, and r = 1 / sqrt(mean x^2 + eps) (1 without a norm).
template <typename F>
struct Turn {
    F C[8], S[8];
    // cs, sn: the row's angles, pair by pair
    template <int D>
    __device__ __forceinline__ void set(const float* weight, int cl, int rotary, bool interleaved, const F* cs, const F* sn) {
        const int reach = rotary / 16;                     // lanes between the two halves of a pair
        const bool turns = 8 * cl < rotary, first = cl < reach;
        const int other = interleaved || !turns ? 8 * cl : 8 * (first ? cl + reach : cl - reach);
        const int pair = !turns ? 0 : (interleaved ? 4 * cl : 8 * (first ? cl : cl - reach));
        F w[8], v[8], c[8], s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
            const float4 a = weight ? *reinterpret_cast<const float4*>(weight + 8 * cl + 4 * h) : one, b = weight ? *reinterpret_cast<const float4*>(weight + other + 4 * h) : one;
            const float4 x = *reinterpret_cast<const float4*>(cs + pair + (interleaved ? 0 : 4 * h)), y = *reinterpret_cast<const float4*>(sn + pair + (interleaved ? 0 : 4 * h));
            w[4 * h] = a.x; w[4 * h + 1] = a.y; w[4 * h + 2] = a.z; w[4 * h + 3] = a.w;
            v[4 * h] = b.x; v[4 * h + 1] = b.y; v[4 * h + 2] = b.z; v[4 * h + 3] = b.w;
            c[4 * h] = x.x; c[4 * h + 1] = x.y; c[4 * h + 2] = x.z; c[4 * h + 3] = x.w;
            s[4 * h] = y.x; s[4 * h + 1] = y.y; s[4 * h + 2] = y.z; s[4 * h + 3] = y.w;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // (interleaved: neighbours share one of the first four pairs that were read)
            const F wp = interleaved ? v[k ^ 1] : v[k], cv = interleaved ? c[k / 2] : c[k], sv = interleaved ? s[k / 2] : s[k];
            const bool minus = interleaved ? !(k & 1) : first;
            C[k] = turns ? w[k] * cv : w[k];
            S[k] = turns ? (minus ? -wp : wp) * sv : (F)-0.0;      // (adds -0 to channels that stay: a zero keeps its sign)
        }
    }
    // x: the lane's channels, y: their partners.  With m: also the sizes |x C| + |x_partner S| times r, which bound what rounding did;
    // the first infinite where the squares have left fp32's range.  In units of 2^-24 of m, what comes before C, S or r is good to: an angle 1, its sine or
    // cosine 4 (two places), the product with w 1; the products with x and their sum 2; r 10.5 (thirteen roundings in the mean, half of which a
    // root passes on, and two places of its own) and its product 1: less than 20, where codes_of_keys allows 32.
    template <int D, bool SIZES = false>
    __device__ __forceinline__ void apply(F (&x)[8], const F (&y)[8], bool norm, float eps, F* m = nullptr) const {
        F r = 1;
        bool lost = false;
        if (norm) {
            F ss = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) ss = fma(x[k], x[k], ss);
#pragma unroll
            for (int s = 1; s < D / 8; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
            const F mean = ss * (F)(1.0 / D) + (F)eps;
            lost = !(mean > (F)1e-30 && mean < (F)1e30);
            r = rsqrt(mean);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (SIZES) {
                const F a = x[k] * C[k], b = y[k] * S[k];
                m[k] = (fabsf(a) + fabsf(b)) * r;
                x[k] = (a + b) * r;
            } else {
                x[k] = fma(x[k], C[k], y[k] * S[k]) * r;
            }
        }
        if constexpr (SIZES) m[0] = lost ? (F)INFINITY : m[0];
    }
};

// ---- Eight channels of a row as codes, and their group's scale, which the lane's neighbour agrees on: scale e4m3(max|x| / (6 g)), codes
// e2m1(x / (scale g)), quotients rounded to fp32.

struct Kv4Codes { uint32_t codes, scale; };

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    unsigned short pair;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(pair) : "f"(hi), "f"(lo));
    return pair;
}
template <typename Q>
__device__ __forceinline__ uint32_t e2m1x8(Q quotient) {
    uint32_t bytes = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) bytes |= f32x2_to_e2m1x2(quotient(2 * k), quotient(2 * k + 1)) << (8 * k);
    return bytes;
}

// As the definition has it, in fp64.
__device__ __forceinline__ Kv4Codes codes_exact(const double (&x)[8], double g) {
    // (rounding is monotonic: the largest of the rounded quotients is the largest quotient rounded)
    const double sixth = 1.0 / (6.0 * g);
    float want = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) want = max_nan(want, fabsf((float)(x[k] * sixth)));
    want = max_nan(want, __shfl_xor_sync(0xffffffffu, want, 1));
    const uint32_t scale = e4m3x2(want, 0.f) & 0xffu;
    const double s = (double)f16_lo(e4m3x2_to_f16x2(scale));
    const bool any = s > 0;                            // (false for a NaN too)
    const double inv = any ? 1.0 / (s * g) : 0.0;
    return {e2m1x8([&](int k) { return any ? (float)(x[k] * inv) : 0.f; }), scale};
}

// Values as they came, where scale * g is exact in fp32 (g of at most 20 significant bits): the quotient correctly rounded from a rounded
// reciprocal and the remainder (Markstein's division), so that ties are ties.  The remainder is taken with its sign turned: that way a zero
// keeps its own.
__device__ __forceinline__ Kv4Codes codes_of_values(const float (&x)[8], float g) {
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max_nan(top, fabsf(x[k]));
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t scale = e4m3x2(__fdiv_rn(top, 6.f * g), 0.f) & 0xffu;
    const float s = f16_lo(e4m3x2_to_f16x2(scale)), sg = s * g;
    const bool any = s > 0.f;
    const float inv = any ? __frcp_rn(sg) : 0.f;
    const uint32_t codes = e2m1x8([&](int k) {
        const float y = x[k] * inv;
        return fabsf(y) < 8.f ? fmaf(-fmaf(y, sg, -x[k]), inv, y) : y;          // (beyond 8, infinities among them, it saturates)
    });
    return {any ? codes : 0u, scale};
}

// Keys in fp32, each off by at most 2^-19 of its m: codes and scale where that cannot change them, else false (for the whole warp).  `touched`: the
// lane's keys were normed or rotated; those that were not are as exact as they came, and divided as values are.
__device__ __forceinline__ bool codes_of_keys(const float (&x)[8], const float (&m)[8], float g, bool touched, Kv4Codes& out) {
    constexpr float OFF = 1.f / (1 << 19), ROUND = 1.f / (1 << 22);
    float top = 0.f, size = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) { top = max_nan(top, fabsf(x[k])); size = fmaxf(size, m[k]); }
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
    size = fmaxf(touched ? size : 0.f, __shfl_xor_sync(0xffffffffu, touched ? size : 0.f, 1));
    const float off = size > 0.f ? fmaf(size, OFF, top * ROUND) : 0.f, six = 6.f * g;
    const uint32_t pair = e4m3x2(__fdiv_rn(top - off, six), __fdiv_rn(top + off, six));
    out.scale = pair & 0xffu;
    const float s = f16_lo(e4m3x2_to_f16x2(out.scale)), sg = s * g;
    const bool any = s > 0.f;
    const float inv = any ? __frcp_rn(sg) : 0.f, off_y = touched ? OFF * inv : 0.f, round_y = touched ? ROUND : 0.f;
    float y[8], e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        y[k] = x[k] * inv;
        y[k] = fabsf(y[k]) < 8.f ? fmaf(-fmaf(y[k], sg, -x[k]), inv, y[k]) : y[k];
        e[k] = fmaf(m[k], off_y, fabsf(y[k]) * round_y);
    }
    // (y + e as the negative of -y - e, whose codes differ in the sign bit: with e = 0 a zero keeps its sign in both)
    out.codes = any ? e2m1x8([&](int k) { return -y[k] - e[k]; }) ^ 0x88888888u : 0u;
    const uint32_t low = any ? e2m1x8([&](int k) { return y[k] - e[k]; }) : 0u;
    return __all_sync(0xffffffffu, top < 1e30f && (pair >> 8) == out.scale && low == out.codes);
}

// Norm and rotation of a lane's keys in fp64.  y: the channels' partners.
template <int D>
__device__ __forceinline__ void turn_exact(const TokensArgs& a, double (&x)[8], const double (&y)[8], int64_t row, int cl) {
    const int reach = a.rotary / 16;
    const bool turns = 8 * cl < a.rotary;
    double ss = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) ss = fma(x[k], x[k], ss);
#pragma unroll
    for (int s = 1; s < D / 8; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
    const double r = a.k_weight ? rsqrt(ss * (1.0 / D) + (double)a.eps) : 1.0;
#pragma unroll 1
    for (int n = 0; n < 8; ++n) {
        const int c = 8 * cl + n, pair = a.interleaved ? c / 2 : (cl < reach ? c : c - a.rotary / 2);
        const int other = a.interleaved ? c ^ 1 : (cl < reach ? c + a.rotary / 2 : c - a.rotary / 2);
        const bool minus = a.interleaved ? !(n & 1) : cl < reach;
        const double w = a.k_weight ? a.k_weight[c] : 1.f, wp = a.k_weight && turns ? a.k_weight[other] : 1.f;
        double cs = 1, sn = 0;
        if (turns) turn_of(a, row, pair, sn, cs);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k == n) x[k] = fma(x[k], w * cs, y[k] * (turns ? (minus ? -wp : wp) * sn : -0.0)) * r;
    }
}

constexpr int TOK_WARPS = 4, TOK_LOADS = 4;       // warps of a CTA; items that a warp has on their way

// Four consecutive channels
template <typename T>
struct Quad {
    uint32_t w[sizeof(T)];
    __device__ __forceinline__ void load(const T* p, bool on) {
        if constexpr (sizeof(T) == 4) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (on) v = __ldcg(reinterpret_cast<const uint4*>(p));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            uint2 v = make_uint2(0, 0);
            if (on) v = __ldcg(reinterpret_cast<const uint2*>(p));
            w[0] = v.x; w[1] = v.y;
        }
    }
    __device__ __forceinline__ void get(float (&x)[4]) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (sizeof(T) == 4) x[k] = __uint_as_float(w[k]);
            else if constexpr (std::is_same<T, __half>::value) x[k] = (k & 1) ? f16_hi(w[k / 2]) : f16_lo(w[k / 2]);
            else x[k] = (k & 1) ? bf16_hi(w[k / 2]) : bf16_lo(w[k / 2]);
        }
    }
};

// A row's queries.  A lane takes four pairs of a head: channels ca .. ca + 3 and their partners cb .. cb + 3 (interleaved: two times two pairs of
// neighbours), so that no channel travels between lanes; y = (x C + x_partner S) r, two channels an instruction.
template <typename T, int D, bool INTER, typename Angles>
__device__ __forceinline__ void queries(const TokensArgs& a, int64_t row, int begin, int end, int lane, const float* cs, const float* sn, Angles angles) {
    constexpr int LPH = D / 8, HPW = 32 / LPH;
    const int hl = lane / LPH, p = 4 * (lane % LPH), half = a.rotary / 2, nq = (a.Hq + HPW - 1) / HPW;
    const bool turns = INTER ? 2 * p < a.rotary : p < half;
    const int ca = INTER ? 2 * p : (turns ? p : half + p), cb = ca + (INTER ? 4 : (turns ? half : D / 2 - half));
    const bool in_last = (nq - 1) * HPW + hl < a.Hq;       // the last item may have fewer heads
    const int64_t step = HPW * a.q_sh;
    const T* from = static_cast<const T*>(a.q) + row * a.q_sr + hl * a.q_sh + begin * step + ca;
    __nv_bfloat16* to = a.q_out + (row * a.Hq + begin * HPW + hl) * D + ca;
    Quad<T> qa[TOK_LOADS], qb[TOK_LOADS];
    auto load = [&](int u, int it) {
        if (it >= end) return;
        const bool on = it < nq - 1 || in_last;
        qa[u].load(from, on);
        qb[u].load(from + (cb - ca), on);
        from += step;
    };
#pragma unroll
    for (int u = 0; u < TOK_LOADS; ++u) load(u, begin + u);
    angles();
    float C[8], S[8];
    {
        const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
        const float4 wa = a.q_weight ? *reinterpret_cast<const float4*>(a.q_weight + ca) : one, wb = a.q_weight ? *reinterpret_cast<const float4*>(a.q_weight + cb) : one;
        const float4 c4 = *reinterpret_cast<const float4*>(cs + p), s4 = *reinterpret_cast<const float4*>(sn + p);
        const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w}, cv[4] = {c4.x, c4.y, c4.z, c4.w}, sv[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int pair = INTER ? k / 2 : k % 4;
            const bool minus = INTER ? !(k & 1) : k < 4;
            const float wp = w[INTER ? k ^ 1 : k ^ 4];
            C[k] = turns ? w[k] * cv[pair] : w[k];
            S[k] = turns ? (minus ? -wp : wp) * sv[pair] : -0.f;
        }
    }
    const bool some_stay = a.rotary < D;
#pragma unroll 1
    for (int it = begin; it < end; it += TOK_LOADS) {
#pragma unroll
        for (int u = 0; u < TOK_LOADS; ++u) {
            if (it + u >= end) break;                  // the same for the whole warp
            float x[8], y[8], r = 1.f;
            {
                float x0[4], x1[4];
                qa[u].get(x0);
                qb[u].get(x1);
#pragma unroll
                for (int k = 0; k < 4; ++k) { x[k] = x0[k]; x[4 + k] = x1[k]; }
            }
            load(u, it + u + TOK_LOADS);
            if (a.q_weight) {
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int k = 0; k < 8; k += 2) fma2(s0, s1, x[k], x[k + 1], x[k], x[k + 1]);
                float ss = s0 + s1;
#pragma unroll
                for (int n = 1; n < LPH; n <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, n);
                r = rsqrtf(ss * (1.f / D) + a.eps);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = x[INTER ? k ^ 1 : k ^ 4];
            if (some_stay && !turns) {                 // channels that do not turn have no part in anything: not even an infinity times 0
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                float t0, t1;
                mul2(t0, t1, y[k], y[k + 1], S[k], S[k + 1]);
                fma2(t0, t1, x[k], x[k + 1], C[k], C[k + 1]);
                mul2(x[k], x[k + 1], t0, t1, r, r);
            }
            if (it + u < nq - 1 || in_last) {
                const uint4 o = pack_bf16(x);
                *reinterpret_cast<uint2*>(to) = make_uint2(o.x, o.y);
                *reinterpret_cast<uint2*>(to + (cb - ca)) = make_uint2(o.z, o.w);
            }
            to += HPW * D;
        }
    }
}

// A warp takes a part of a row's queries, or of its keys and values, an item (two or four heads) after the other, four on their way at any time.
template <typename T, int D, bool KV4>
__global__ void __launch_bounds__(32 * TOK_WARPS, sizeof(T) == 4 ? 4 : 5) append_tokens_kernel(const __grid_constant__ TokensArgs a) {
    constexpr int LPH = D / 8, HPW = 32 / LPH;         // lanes of a head, heads of a warp
    __shared__ __align__(16) float s_cos[2][D / 2], s_sin[2][D / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // two rows with two warps each, or four warps of the 4 * ctas_row that a row has
    const bool two = a.ctas_row == 0;
    int row, part;
    if (two) { row = blockIdx.x * 2 + (warp >> 1); part = warp & 1; }
    else { a.div_ctas.divmod((int)blockIdx.x, row, part); part = 4 * part + warp; }
    const int tab = two ? warp >> 1 : 0, sub = two ? threadIdx.x & 63 : threadIdx.x, others_by = two ? 64 : 128;
    float *const cs = s_cos[tab], *const sn = s_sin[tab];
    pdl_wait();
    const int64_t slot = row < a.rows ? (int64_t)__ldcg(reinterpret_cast<const long long*>(a.slot_map) + row) : -1;
    const bool live = slot >= 0 && slot < a.limit;
    // the row's angles, by all its warps of the CTA: every warp of a CTA comes here once
    auto angles = [&]() {
        if (a.rotary && live)
            for (int c = sub; c < a.rotary / 2; c += others_by) turn_of(a, row, c, sn[c], cs[c]);
        __syncthreads();
    };
    if (!live) {
        if (slot >= 0 && lane == 0 && part == 0 && a.status) atomicOr(a.status, ETA_DEV_BAD_SLOT);
        angles();
        return;
    }
    if (part < a.q_parts) {
        const int nq = (a.Hq + HPW - 1) / HPW, begin = part * nq / a.q_parts, end = (part + 1) * nq / a.q_parts;
        if (a.interleaved) queries<T, D, true>(a, row, begin, end, lane, cs, sn, angles);
        else queries<T, D, false>(a, row, begin, end, lane, cs, sn, angles);
        return;
    }
    // ---- keys, then values: a lane holds eight consecutive channels, so that two lanes hold a group of the 4-bit cache
    const int nkv = (a.Hkv + HPW - 1) / HPW, begin = (part - a.q_parts) * 2 * nkv / a.kv_parts, end = (part - a.q_parts + 1) * 2 * nkv / a.kv_parts;
    const int hl = lane / LPH, cl = lane % LPH;
    const bool in_last = (nkv - 1) * HPW + hl < a.Hkv;     // the last item may have fewer heads
    int64_t page;
    int off;
    if (a.limit <= INT32_MAX) { int p32; a.div_page.divmod((int)slot, p32, off); page = p32; }
    else { page = slot / a.per_page; off = (int)(slot - page * a.per_page); }
    // items first .. last - 1 of a tensor, four on their way: use(piece, item, whether the lane has a head of it)
    auto stream = [&](const void* tensor, int64_t sr, int64_t sh, int first, int last, auto&& ready, auto&& use) {
        const T* from = static_cast<const T*>(tensor) + (int64_t)row * sr + (first * HPW + hl) * sh + 8 * cl;
        const int64_t step = HPW * sh;
        Piece<T> pc[TOK_LOADS];
        auto load = [&](int u, int it) {
            if (it >= last) return;
            pc[u].load(from, it < nkv - 1 || in_last);
            from += step;
        };
#pragma unroll
        for (int u = 0; u < TOK_LOADS; ++u) load(u, first + u);
        ready();
#pragma unroll 1
        for (int it = first; it < last; it += TOK_LOADS) {
#pragma unroll
            for (int u = 0; u < TOK_LOADS; ++u) {
                if (it + u >= last) break;                 // the same for the whole warp
                const Piece<T> now = pc[u];
                load(u, it + u + TOK_LOADS);
                use(now, it + u, it + u < nkv - 1 || in_last);
            }
        }
    };
    // the pairs' other halves are in lane `partner`, or in the lane's own neighbours
    const int reach = a.rotary / 16;
    const bool turns = 8 * cl < a.rotary;
    const int partner = a.interleaved || !turns ? lane : (cl < reach ? lane + reach : lane - reach);
    auto others = [&](const Piece<T>& p, auto& y) {
        Piece<T> o = p;
        if (a.rotary && !a.interleaved) o.exchange(partner);
        o.get(y);
        if (a.interleaved) {
#pragma unroll
            for (int c = 0; c < 8; c += 2) { const auto t = y[c]; y[c] = y[c + 1]; y[c + 1] = t; }
        }
        if (a.rotary < D && !turns) {
#pragma unroll
            for (int c = 0; c < 8; ++c) y[c] = 0;
        }
    };
    const int k0 = min(begin, nkv), k1 = min(end, nkv), v0 = max(begin, nkv) - nkv, v1 = max(end, nkv) - nkv;
    Turn<float> turn;
    auto turned = [&]() {
        angles();
        if (k0 < k1) turn.template set<D>(a.k_weight, cl, a.rotary, a.interleaved != 0, cs, sn);
    };
    auto nothing = []() {};
    if constexpr (!KV4) {
        const int64_t kb = page * a.ks_b + (int64_t)off * a.ks_t + 8 * cl, vb = page * a.vs_b + (int64_t)off * a.vs_t + 8 * cl;
        stream(a.k, a.k_sr, a.k_sh, k0, k1, turned, [&](const Piece<T>& p, int it, bool on) {
            float x[8], y[8];
            p.get(x);
            others(p, y);
            turn.template apply<D>(x, y, a.k_weight != nullptr, a.eps);
            if (on) *reinterpret_cast<uint4*>(a.K + kb + (it * HPW + hl) * a.ks_h) = pack_bf16(x);
        });
        stream(a.v, a.v_sr, a.v_sh, v0, v1, nothing, [&](const Piece<T>& p, int it, bool on) {
            float x[8];
            p.get(x);
            if (on) *reinterpret_cast<uint4*>(a.V + vb + (it * HPW + hl) * a.vs_h) = pack_bf16(x);
        });
    } else {
        // this row's codes in a head's block: byte of the codes, and of the scale that the pair of lanes holds
        const int b_shift = a.b == 32 ? 5 : (a.b == 64 ? 6 : 7), t = off & (a.b - 1);
        unsigned char* const base = a.pool + page * a.ks_b + (int64_t)(off >> b_shift) * a.ks_t;
        const int c_at = t * (D / 2) + 4 * cl, s_at = a.b * (D / 2) + t * (D / KV4_GROUP) + cl / 2;
        auto store = [&](const Kv4Codes& c, int tensor_at, int it) {
            unsigned char* const to = base + (it * HPW + hl) * a.ks_h + tensor_at;
            *reinterpret_cast<uint32_t*>(to + c_at) = c.codes;
            if ((cl & 1) == 0) to[s_at] = (unsigned char)c.scale;
        };
        const int v_at = Kv4Block(a.b, D).v_codes;
        uint64_t left = 0;                                 // keys that fp32 did not settle (bit 63: one of those from there on)
        stream(a.k, a.k_sr, a.k_sh, k0, k1, turned, [&](const Piece<T>& p, int it, bool on) {
            float x[8], y[8], m[8];
            p.get(x);
            others(p, y);
            turn.template apply<D, true>(x, y, a.k_weight != nullptr, a.eps, m);
            Kv4Codes c;
            if (codes_of_keys(x, m, a.k_scale, turns || a.k_weight, c) && (a.fast & 1)) {
                if (on) store(c, 0, it);
            } else {
                left |= 1ull << min(it - k0, 63);
            }
        });
        if (a.fast & 2) {
            stream(a.v, a.v_sr, a.v_sh, v0, v1, nothing, [&](const Piece<T>& p, int it, bool on) {
                float x[8];
                p.get(x);
                const Kv4Codes c = codes_of_values(x, a.v_scale);
                if (on) store(c, v_at, it);
            });
        } else {
            stream(a.v, a.v_sr, a.v_sh, v0, v1, nothing, [&](const Piece<T>& p, int it, bool on) {
                double x[8];
                p.get(x);
                const Kv4Codes c = codes_exact(x, a.v_scale);
                if (on) store(c, v_at, it);
            });
        }
        // what lies too near a border between two codes for fp32, about one item in a hundred, once more in fp64
        for (int it = k0; left != 0 && it < k1; ++it) {
            if (((left >> min(it - k0, 63)) & 1) == 0) continue;
            const bool on = it < nkv - 1 || in_last;
            Piece<T> p;
            p.load(static_cast<const T*>(a.k) + (int64_t)row * a.k_sr + (it * HPW + hl) * a.k_sh + 8 * cl, on);
            double x[8], y[8];
            p.get(x);
            others(p, y);
            turn_exact<D>(a, x, y, row, cl);
            const Kv4Codes c = codes_exact(x, a.k_scale);
            if (on) store(c, 0, it);
        }
    }
}

// A thread per group of sixteen channels: 9 bytes in, 32 out.
struct UnpackArgs {
    const unsigned char* pool;
    int64_t sb, sh, sj;
    float k_scale, v_scale;
    int Hkv, b, nb, t_end;
    int64_t groups;
    __nv_bfloat16 *K, *V;
    int64_t ks_b, ks_h, ks_t, vs_b, vs_h, vs_t;
};
template <int D>
__global__ void __launch_bounds__(256) unpack_kv4_kernel(const UnpackArgs a) {
    constexpr int GPT = D / KV4_GROUP;                 // groups of a token
    pdl_wait();
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= a.groups) return;
    // block after block (sequence or page, head, block of the sequence), K then V, token after token
    const int b = a.b, per_block = 2 * b * GPT;
    const int64_t blk = n / per_block;
    int m = (int)(n - blk * per_block);
    const bool is_v = m >= b * GPT;
    if (is_v) m -= b * GPT;
    const int t = m / GPT, gr = m % GPT;
    const int j = (int)(blk % a.nb), hk = (int)(blk / a.nb % a.Hkv);
    const int64_t i = blk / a.nb / a.Hkv, tok = (int64_t)j * b + t;
    if (tok >= a.t_end) return;
    const unsigned char* from = a.pool + i * a.sb + hk * a.sh + j * a.sj + (is_v ? Kv4Block(b, D).v_codes : 0);
    const uint2 codes = __ldcg(reinterpret_cast<const uint2*>(from + t * (D / 2)) + gr);
    const float s = f16_lo(e4m3x2_to_f16x2(__ldcg(from + b * (D / 2) + t * GPT + gr))) * (is_v ? a.v_scale : a.k_scale);
    __nv_bfloat16* to = (is_v ? a.V + i * a.vs_b + hk * a.vs_h + tok * a.vs_t : a.K + i * a.ks_b + hk * a.ks_h + tok * a.ks_t) + gr * 16;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t w = half ? codes.y : codes.x;
        uint32_t p[4];
        float x[8];
        e2m1x8_to_f16x2(w, p);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[2 * k] = f16_lo(p[k]) * s;
            x[2 * k + 1] = f16_hi(p[k]) * s;
        }
        reinterpret_cast<uint4*>(to)[half] = pack_bf16(x);
    }
}

// ------------------------------------------------------------------ host side

int validate_kv4(const eta_cache_desc* d, const eta_kv4_desc* kv4, const void* pool, bool paged) {
    if (!kv4 || !pool) return ETA_ERR_INVALID_ARG;
    if (!(kv4->k_scale > 0.f) || !(kv4->v_scale > 0.f) || !isfinite(kv4->k_scale) || !isfinite(kv4->v_scale)) return ETA_ERR_INVALID_ARG;
    if (((kv4->stride_b | kv4->stride_h | (paged ? 0 : kv4->stride_j)) & 15) || (reinterpret_cast<uintptr_t>(pool) & 15))
        return ETA_ERR_UNSUPPORTED;
    const int64_t bytes = Kv4Block(d->block_size, d->head_dim).bytes;
    if (kv4->stride_b < bytes || kv4->stride_h < bytes || (!paged && kv4->stride_j < bytes)) return ETA_ERR_INVALID_ARG;
    return ETA_OK;
}

static bool misaligned(std::initializer_list<const void*> pointers, uintptr_t to) {
    for (const void* p : pointers)
        if (reinterpret_cast<uintptr_t>(p) & (to - 1)) return true;
    return false;
}

// eta_append_tokens, and with `kv4` eta_append_tokens_kv4 (K is the pool then)
static int append_tokens(const eta_cache_desc* desc, const eta_kv4_desc* kv4, const eta_tokens_desc* tok, const void* q, const void* k,
                         const void* v, const float* q_weight, const float* k_weight, const double* inv_freq, const int32_t* positions,
                         const int64_t* slot_map, int32_t n_pages, void* q_out, void* K, void* V, uint32_t* status, void* stream) {
    int rc = validate_shape(desc);
    if (rc != ETA_OK) return rc;
    if (!tok || tok->n_rows < 0 || n_pages < 0 || tok->type < ETA_TYPE_BF16 || tok->type > ETA_TYPE_FP32) return ETA_ERR_INVALID_ARG;
    if ((tok->flags & ~ETA_TOKENS_INTERLEAVED) || !(tok->eps >= 0.f)) return ETA_ERR_INVALID_ARG;
    if (tok->rotary_dim < 0 || tok->rotary_dim > desc->head_dim) return ETA_ERR_INVALID_ARG;
    if (tok->rotary_dim % 16) return ETA_ERR_UNSUPPORTED;
    if ((rc = kv4 ? validate_kv4(desc, kv4, K, n_pages > 0) : validate_strides(desc)) != ETA_OK) return rc;
    if (!q || !k || !v || !slot_map || !q_out || !K || !V) return ETA_ERR_INVALID_ARG;
    if (tok->rotary_dim && (!inv_freq || !positions)) return ETA_ERR_INVALID_ARG;
    const int64_t vec = tok->type == ETA_TYPE_FP32 ? 4 : 8;
    for (int64_t stride : {tok->q_stride_r, tok->q_stride_h, tok->k_stride_r, tok->k_stride_h, tok->v_stride_r, tok->v_stride_h})
        if (stride % vec) return ETA_ERR_UNSUPPORTED;
    if (misaligned({q, k, v, q_out, K, V, q_weight, k_weight}, 16) || misaligned({slot_map, inv_freq}, 8) || misaligned({positions}, 4))
        return ETA_ERR_UNSUPPORTED;
    if (tok->n_rows == 0) return ETA_OK;
    if (tok->n_rows > (1 << 30)) return ETA_ERR_UNSUPPORTED;

    TokensArgs a;
    a.q = q; a.k = k; a.v = v;
    a.q_weight = q_weight; a.k_weight = k_weight; a.inv_freq = inv_freq; a.positions = positions; a.slot_map = slot_map;
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.K = static_cast<__nv_bfloat16*>(K); a.V = static_cast<__nv_bfloat16*>(V);
    a.pool = static_cast<unsigned char*>(K);
    a.status = status;
    a.q_sr = tok->q_stride_r; a.q_sh = tok->q_stride_h; a.k_sr = tok->k_stride_r; a.k_sh = tok->k_stride_h;
    a.v_sr = tok->v_stride_r; a.v_sh = tok->v_stride_h;
    a.ks_b = desc->k_stride_b; a.ks_h = desc->k_stride_h; a.ks_t = desc->k_stride_t;
    a.vs_b = desc->v_stride_b; a.vs_h = desc->v_stride_h; a.vs_t = desc->v_stride_t;
    if (kv4) { a.ks_b = kv4->stride_b; a.ks_h = kv4->stride_h; a.ks_t = n_pages > 0 ? 0 : kv4->stride_j; }
    a.k_scale = kv4 ? kv4->k_scale : 1; a.v_scale = kv4 ? kv4->v_scale : 1;
    const auto plain = [](float g) {
        uint32_t bits;
        memcpy(&bits, &g, 4);
        return g >= 0x1p-60f && g <= 0x1p60f && (bits & 0xfu) == 0;
    };
    a.fast = (plain(a.k_scale) ? 1 : 0) | (plain(a.v_scale) ? 2 : 0);
    a.per_page = n_pages > 0 ? desc->block_size : desc->t_cap;
    a.limit = (int64_t)a.per_page * (n_pages > 0 ? n_pages : desc->batch);
    a.rows = tok->n_rows; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads; a.b = desc->block_size;
    a.rotary = tok->rotary_dim; a.interleaved = (tok->flags & ETA_TOKENS_INTERLEAVED) != 0;
    a.eps = tok->eps;
    a.div_page = FastDiv(a.per_page);
    // Two warps to a row, one for its queries, one for its keys and values, where there are rows enough to fill the GPU (148 SMs; a partition of it only
    // gets more CTAs than it needs); as many as there are items where there are not.
    const int per_warp = 32 / (desc->head_dim / 8);
    const int q_items = (a.Hq + per_warp - 1) / per_warp, kv_items = 2 * ((a.Hkv + per_warp - 1) / per_warp);
    const int want = (148 * 16 / 4 + a.rows - 1) / a.rows, most = (q_items + kv_items + 3) / 4;
    a.ctas_row = a.rows >= 148 * 8 ? 0 : (want > most ? most : want);
    const int parts = a.ctas_row ? 4 * a.ctas_row : 2;
    a.kv_parts = parts / 2 < kv_items ? parts / 2 : kv_items;
    a.q_parts = parts - a.kv_parts;
    a.div_ctas = FastDiv(a.ctas_row ? a.ctas_row : 1);
    const unsigned ctas = a.ctas_row ? (unsigned)a.rows * a.ctas_row : ((unsigned)a.rows + 1) / 2;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const char* what = kv4 ? "eta_append_tokens_kv4" : "eta_append_tokens";
#define ETA_TOK(T, DD, Q4) launch_pdl(what, append_tokens_kernel<T, DD, Q4>, dim3(ctas), dim3(32 * TOK_WARPS), 0, s, a)
#define ETA_TOK_D(T) (desc->head_dim == 128 ? (kv4 ? ETA_TOK(T, 128, true) : ETA_TOK(T, 128, false)) : (kv4 ? ETA_TOK(T, 64, true) : ETA_TOK(T, 64, false)))
    return tok->type == ETA_TYPE_BF16 ? ETA_TOK_D(__nv_bfloat16) : (tok->type == ETA_TYPE_FP16 ? ETA_TOK_D(__half) : ETA_TOK_D(float));
#undef ETA_TOK_D
#undef ETA_TOK
}

}  // namespace eta

extern "C" {

size_t eta_kv4_block_bytes(int32_t block_size, int32_t head_dim) {
    if ((block_size != 32 && block_size != 64 && block_size != 128) || (head_dim != 64 && head_dim != 128)) return 0;
    return (size_t)eta::Kv4Block(block_size, head_dim).bytes;
}

int eta_append_tokens(const eta_cache_desc* desc, const eta_tokens_desc* tokens, const void* q, const void* k, const void* v,
                      const float* q_weight, const float* k_weight, const double* inv_freq, const int32_t* positions,
                      const int64_t* slot_map, int32_t n_pages, void* q_out, void* K, void* V, uint32_t* status_dev, void* stream) {
    return eta::append_tokens(desc, nullptr, tokens, q, k, v, q_weight, k_weight, inv_freq, positions, slot_map, n_pages, q_out, K, V,
                              status_dev, stream);
}

int eta_append_tokens_kv4(const eta_cache_desc* desc, const eta_kv4_desc* kv4, const eta_tokens_desc* tokens, const void* q,
                          const void* k, const void* v, const float* q_weight, const float* k_weight, const double* inv_freq,
                          const int32_t* positions, const int64_t* slot_map, int32_t n_pages, void* q_out, void* pool,
                          uint32_t* status_dev, void* stream) {
    if (!kv4) return ETA_ERR_INVALID_ARG;
    return eta::append_tokens(desc, kv4, tokens, q, k, v, q_weight, k_weight, inv_freq, positions, slot_map, n_pages, q_out, pool, pool,
                              status_dev, stream);
}

int eta_unpack_kv4(const eta_cache_desc* desc, const eta_kv4_desc* kv4, const void* pool, int32_t n_pages, void* K, void* V, void* stream) {
    using namespace eta;
    int rc = validate_shape(desc);
    if (rc != ETA_OK) return rc;
    if (n_pages < 0 || !K || !V) return ETA_ERR_INVALID_ARG;
    if ((rc = validate_kv4(desc, kv4, pool, n_pages > 0)) != ETA_OK || (rc = validate_strides(desc)) != ETA_OK) return rc;
    if (misaligned({K, V}, 16)) return ETA_ERR_UNSUPPORTED;
    UnpackArgs a;
    a.pool = static_cast<const unsigned char*>(pool);
    a.sb = kv4->stride_b; a.sh = kv4->stride_h; a.sj = n_pages > 0 ? 0 : kv4->stride_j;
    a.k_scale = kv4->k_scale; a.v_scale = kv4->v_scale;
    a.Hkv = desc->n_kv_heads; a.b = desc->block_size;
    a.t_end = n_pages > 0 ? a.b : desc->t_cap;
    a.nb = (int)(((int64_t)a.t_end + a.b - 1) / a.b);
    a.groups = (int64_t)(n_pages > 0 ? n_pages : desc->batch) * a.Hkv * a.nb * 2 * a.b * (desc->head_dim / KV4_GROUP);
    a.K = static_cast<__nv_bfloat16*>(K); a.V = static_cast<__nv_bfloat16*>(V);
    a.ks_b = desc->k_stride_b; a.ks_h = desc->k_stride_h; a.ks_t = desc->k_stride_t;
    a.vs_b = desc->v_stride_b; a.vs_h = desc->v_stride_h; a.vs_t = desc->v_stride_t;
    const int64_t ctas = (a.groups + 255) / 256;
    if (ctas > INT32_MAX) return ETA_ERR_UNSUPPORTED;
    return launch_pdl("eta_unpack_kv4", desc->head_dim == 128 ? unpack_kv4_kernel<128> : unpack_kv4_kernel<64>, dim3((unsigned)ctas), dim3(256), 0,
                      static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"
