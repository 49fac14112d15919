// New tokens of a step: norm of every query and key head, rotation by position, the queries stored for the step and the keys and
// values written to the cache, bf16 or 4-bit, in one pass over the projections; and a 4-bit cache read back as a bf16 one.
//
//   y = x * w / sqrt(mean_c x_c^2 + eps);   (a, b) -> (a cos - b sin, a sin + b cos),  angle = position * inv_freq
//
// A warp takes one row's heads two (d = 128) or four (64) at a time, a piece of eight channels per lane: a head's sum and a channel's
// partner are shuffles away, and everything is read once and written once.
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
    int rows, Hq, Hkv, per_page, b, parts, rotary, interleaved;
    float k_scale, v_scale;
    int fast;              // bit 0: the keys' scale is of a size that leaves fp32 its range; bit 1: the values' too, and its product with a group's is exact
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

// The angle of a row's pair, reduced by whole turns with a two-part 2 pi (Cody and Waite): any 32-bit position keeps its 64-bit angle
__device__ __forceinline__ double reduced_angle(const TokensArgs& a, int64_t row, int pair) {
    const double x = (double)__ldcg(a.positions + row) * __ldcg(a.inv_freq + pair), n = rint(x * 0.15915494309189535);
    return fma(-n, 2.4492935982947064e-16, fma(-n, 6.283185307179586, x));
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
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = 8 * cl + k, other = interleaved ? c ^ 1 : (first ? c + rotary / 2 : c - rotary / 2);
            const int pair = interleaved ? c / 2 : (first ? c : c - rotary / 2);
            const bool minus = interleaved ? !(k & 1) : first;
            const F w = weight ? (F)weight[c] : (F)1, wp = weight && turns ? (F)weight[other] : (F)1;
            C[k] = turns ? w * cs[pair] : w;
            S[k] = turns ? (minus ? -wp : wp) * sn[pair] : (F)0;
        }
    }
    // x: the lane's channels, y: their partners.  With m: also the sizes |x C| + |x_partner S| times r, which bound what rounding did.
    template <int D, bool SIZES = false>
    __device__ __forceinline__ void apply(F (&x)[8], const F (&y)[8], bool norm, float eps, F* m = nullptr) const {
        F r = 1;
        if (norm) {
            F ss = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) ss = fma(x[k], x[k], ss);
#pragma unroll
            for (int s = 1; s < D / 8; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
            r = rsqrt(ss * (F)(1.0 / D) + (F)eps);
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
// reciprocal and the remainder (Markstein's division), so that ties are ties.
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
        return fabsf(y) < 8.f ? fmaf(fmaf(-y, sg, x[k]), inv, y) : y;          // (beyond 8, infinities among them, it saturates)
    });
    return {any ? codes : 0u, scale};
}

// Keys in fp32, each off by at most 2^-19 of its m: codes and scale where that cannot change them, else false (for the whole warp).
__device__ __forceinline__ bool codes_of_keys(const float (&x)[8], const float (&m)[8], float g, Kv4Codes& out) {
    constexpr float OFF = 1.f / (1 << 19), ROUND = 1.f / (1 << 22);
    float top = 0.f, size = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) { top = max_nan(top, fabsf(x[k])); size = fmaxf(size, m[k]); }
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
    size = fmaxf(size, __shfl_xor_sync(0xffffffffu, size, 1));
    const float sixth = 1.f / (6.f * g), off = size * OFF + top * ROUND;
    const uint32_t pair = e4m3x2((top - off) * sixth, (top + off) * sixth);
    out.scale = pair & 0xffu;
    const float s = f16_lo(e4m3x2_to_f16x2(out.scale));
    const float inv = s > 0.f ? rcp_approx(s * g) : 0.f;
    float e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) e[k] = fmaf(m[k], OFF * inv, fabsf(x[k] * inv) * ROUND);
    out.codes = e2m1x8([&](int k) { return fmaf(x[k], inv, e[k]); });
    const uint32_t low = e2m1x8([&](int k) { return fmaf(x[k], inv, -e[k]); });
    return __all_sync(0xffffffffu, top < 1e30f && (pair >> 8) == out.scale && low == out.codes);
}

// Token t of a tensor's codes and scales at `to`, in a block of b
__device__ __forceinline__ void store_codes(const Kv4Codes& c, unsigned char* to, int b, int D, int t, int cl) {
    *reinterpret_cast<uint32_t*>(to + t * (D / 2) + 4 * cl) = c.codes;
    if ((cl & 1) == 0) to[b * (D / 2) + t * (D / KV4_GROUP) + cl / 2] = (unsigned char)c.scale;
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
        if (turns) sincos(reduced_angle(a, row, pair), &sn, &cs);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k == n) x[k] = fma(x[k], w * cs, y[k] * ((minus ? -wp : wp) * sn)) * r;
    }
}

constexpr int TOK_WARPS = 4, TOK_LOADS = 4;       // warps of a CTA; pieces that a lane has in flight

// A warp takes items (two or four heads of the row each) one after the other, four on their way at any time: queries, keys, values.
template <typename T, int D, bool KV4>
__global__ void __launch_bounds__(32 * TOK_WARPS, sizeof(T) == 4 ? 4 : 5) append_tokens_kernel(const __grid_constant__ TokensArgs a) {
    constexpr int LPH = D / 8, HPW = 32 / LPH;         // lanes of a head, heads of a warp
    __shared__ float s_cos[TOK_WARPS][D / 2], s_sin[TOK_WARPS][D / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    const int64_t wid = (int64_t)blockIdx.x * TOK_WARPS + warp;
    const int64_t row = wid / a.parts;
    const int part = (int)(wid % a.parts);
    if (row >= a.rows) return;
    const int64_t slot = __ldcg(reinterpret_cast<const long long*>(a.slot_map) + row);
    if (slot < 0) return;
    if (slot >= a.limit) {
        if (lane == 0 && part == 0 && a.status) atomicOr(a.status, ETA_DEV_BAD_SLOT);
        return;
    }
    const int nq = (a.Hq + HPW - 1) / HPW, nkv = (a.Hkv + HPW - 1) / HPW, all = nq + 2 * nkv;
    const int begin = part * all / a.parts, end = (part + 1) * all / a.parts;
    const int hl = lane / LPH, cl = lane % LPH;
    const T *const q = static_cast<const T*>(a.q) + row * a.q_sr + 8 * cl, *const k = static_cast<const T*>(a.k) + row * a.k_sr + 8 * cl,
            *const v = static_cast<const T*>(a.v) + row * a.v_sr + 8 * cl;
    Piece<T> pc[TOK_LOADS];
    auto load = [&](Piece<T>& p, int it) {
        const bool is_q = it < nq, is_k = it < nq + nkv;
        const int head = (is_q ? it : (is_k ? it - nq : it - nq - nkv)) * HPW + hl;
        p.load(is_q ? q + head * a.q_sh : (is_k ? k + head * a.k_sh : v + head * a.v_sh), it < end && head < (is_q ? a.Hq : a.Hkv));
    };
#pragma unroll
    for (int u = 0; u < TOK_LOADS; ++u) load(pc[u], begin + u);
    // ---- the row's angles
    if (a.rotary && begin < nq + nkv) {
        for (int c = lane; c < a.rotary / 2; c += 32) sincosf((float)reduced_angle(a, row, c), &s_sin[warp][c], &s_cos[warp][c]);
        __syncwarp();
    }
    const int64_t page = slot / a.per_page;
    const int off = (int)(slot - page * a.per_page);
    // the pairs' other halves are in lane `partner`, or in the lane's own neighbours
    const int reach = a.rotary / 16;
    const int partner = a.interleaved || 8 * cl >= a.rotary ? lane : (cl < reach ? lane + reach : lane - reach);
    auto others = [&](const Piece<T>& p, auto& y) {
        Piece<T> o = p;
        if (a.rotary && !a.interleaved) o.exchange(partner);
        o.get(y);
        if (a.interleaved) {
#pragma unroll
            for (int c = 0; c < 8; c += 2) { const auto t = y[c]; y[c] = y[c + 1]; y[c + 1] = t; }
        }
        if (a.rotary < D && 8 * cl >= a.rotary) {      // channels that do not turn have no part in anything: not even an infinity times 0
#pragma unroll
            for (int c = 0; c < 8; ++c) y[c] = 0;
        }
    };
    Turn<float> turn;
    if (begin < nq) turn.template set<D>(a.q_weight, cl, a.rotary, a.interleaved != 0, s_cos[warp], s_sin[warp]);
    // ---- queries
    int it = begin;
    for (; it < end && it < nq; it += TOK_LOADS) {
#pragma unroll
        for (int u = 0; u < TOK_LOADS; ++u) {
            if (it + u < end && it + u < nq) {         // the same for the whole warp
                float x[8], y[8];
                pc[u].get(x);
                others(pc[u], y);
                load(pc[u], it + u + TOK_LOADS);
                turn.template apply<D>(x, y, a.q_weight != nullptr, a.eps);
                const int head = (it + u) * HPW + hl;
                if (head < a.Hq) *reinterpret_cast<uint4*>(a.q_out + (row * a.Hq + head) * D + 8 * cl) = pack_bf16(x);
            }
        }
    }
    // where a head's codes of this row's block are
    auto place = [&](bool is_k, int head) {
        return a.pool + page * a.ks_b + head * a.ks_h + (int64_t)(off / a.b) * a.ks_t + (is_k ? 0 : Kv4Block(a.b, D).v_codes);
    };
    uint64_t left = 0;                                 // items that fp32 did not settle (bit 63: one of those from there on)
    // ---- keys and values
    const int first = max(begin, nq);                  // pieces of these items are in the slots that follow the queries'
    if (first < end && first < nq + nkv) turn.template set<D>(a.k_weight, cl, a.rotary, a.interleaved != 0, s_cos[warp], s_sin[warp]);
    for (it = first - (first - begin) % TOK_LOADS; it < end; it += TOK_LOADS) {
#pragma unroll
        for (int u = 0; u < TOK_LOADS; ++u) {
            if (it + u >= first && it + u < end) {
                const bool is_k = it + u < nq + nkv;
                const int head = (is_k ? it + u - nq : it + u - nq - nkv) * HPW + hl;
                const bool on = head < a.Hkv;
                float x[8], y[8];
                pc[u].get(x);
                if (is_k) others(pc[u], y);
                load(pc[u], it + u + TOK_LOADS);
                if constexpr (KV4) {
                    Kv4Codes c;
                    bool settled;
                    if (is_k) {
                        float m[8];
                        turn.template apply<D, true>(x, y, a.k_weight != nullptr, a.eps, m);
                        settled = codes_of_keys(x, m, a.k_scale, c) && (a.fast & 1);
                    } else {
                        c = codes_of_values(x, a.v_scale);
                        settled = (a.fast & 2) != 0;
                    }
                    if (settled) {
                        if (on) store_codes(c, place(is_k, head), a.b, D, off % a.b, cl);
                    } else {
                        left |= 1ull << min(it + u - first, 63);
                    }
                } else {
                    if (is_k) turn.template apply<D>(x, y, a.k_weight != nullptr, a.eps);
                    __nv_bfloat16* to = is_k ? a.K + page * a.ks_b + head * a.ks_h + off * a.ks_t : a.V + page * a.vs_b + head * a.vs_h + off * a.vs_t;
                    if (on) *reinterpret_cast<uint4*>(to + 8 * cl) = pack_bf16(x);
                }
            }
        }
    }
    if constexpr (KV4) {
        // ---- what lies too near a border between two codes for fp32, about one item in a hundred, once more in fp64
        for (it = first; left != 0 && it < end; ++it) {
            if (((left >> min(it - first, 63)) & 1) == 0) continue;
            const bool is_k = it < nq + nkv;
            const int head = (is_k ? it - nq : it - nq - nkv) * HPW + hl;
            double x[8], y[8];
            load(pc[0], it);
            pc[0].get(x);
            if (is_k) {
                others(pc[0], y);
                turn_exact<D>(a, x, y, row, cl);
            }
            const Kv4Codes c = codes_exact(x, is_k ? a.k_scale : a.v_scale);
            if (head < a.Hkv) store_codes(c, place(is_k, head), a.b, D, off % a.b, cl);
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
    const auto plain_size = [](float g) { return g >= 0x1p-60f && g <= 0x1p60f; };
    uint32_t v_bits;
    memcpy(&v_bits, &a.v_scale, 4);
    a.fast = (plain_size(a.k_scale) ? 1 : 0) | (plain_size(a.v_scale) && (v_bits & 0xfu) == 0 ? 2 : 0);
    a.per_page = n_pages > 0 ? desc->block_size : desc->t_cap;
    a.limit = (int64_t)a.per_page * (n_pages > 0 ? n_pages : desc->batch);
    a.rows = tok->n_rows; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads; a.b = desc->block_size;
    a.rotary = tok->rotary_dim; a.interleaved = (tok->flags & ETA_TOKENS_INTERLEAVED) != 0;
    a.eps = tok->eps;
    // A row is one warp's work where there are rows enough to fill the GPU, and split as far as it goes where there are not.
    const int per_warp = 32 / (desc->head_dim / 8);
    const int items = (a.Hq + per_warp - 1) / per_warp + 2 * ((a.Hkv + per_warp - 1) / per_warp);
    const int64_t want = ((int64_t)148 * 16 + a.rows - 1) / a.rows;
    a.parts = (int)(want > items ? items : want);
    const int64_t ctas = ((int64_t)a.rows * a.parts + TOK_WARPS - 1) / TOK_WARPS;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const char* what = kv4 ? "eta_append_tokens_kv4" : "eta_append_tokens";
#define ETA_TOK(T, DD, Q4) launch_pdl(what, append_tokens_kernel<T, DD, Q4>, dim3((unsigned)ctas), dim3(32 * TOK_WARPS), 0, s, a)
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
