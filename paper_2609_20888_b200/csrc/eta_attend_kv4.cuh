// Gated attention of one KV head's query heads over a block of a 4-bit cache in shared memory, by a group of four warps: what Attend
// (eta_attend.cuh) is for bf16 tiles, with the same gate, masks and statistics.
//
// A quarter of the bytes per token leaves a quarter of the time per token, so the work per token is what has to be small:
//   - tokens are the rows of the first product (S = K q^T: sixteen tokens an MMA, query heads its eight columns), channels the rows of the second
//     (O^T = V^T P), so that no row of an MMA is padding; the probabilities get from one's layout to the other's by a transpose of 8x8.
//   - a code is converted by the hardware, two at a time, and scaled as an fp16 pair: code * scale is exact in fp16, so both products are
//     exact and their sums fp32.  Queries are scaled by a power of two per head to use fp16's range (their bf16 values stay exact
//     down to 2^-38 of the head's largest).
//   - probabilities are fed as an fp16 value and an fp16 remainder (22 bits).  Up to four heads, both are columns of one MMA: columns 4 to 7
//     repeat the heads of 0 to 3, whose lanes compute the same scores again and feed the remainder.
//   - the running maximum follows the scores only when one is more than SLACK above it: exp(s - m) is then at most 2^2, and with
//     the factor 2^BASE, which every part carries and the final division drops, inside fp16's range at both ends.
#pragma once

#include "eta_attend.cuh"
#include "eta_kv4.cuh"

namespace eta {

__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr) {
    unsigned short v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
// 8x8 matrix of 16-bit elements, two neighbours of a row per lane: transposed
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// One warp's part: tokens warp * WT .. of a block of TS.  Lane (g, t) = (lane / 4, lane % 4) holds the scores of tokens g and g + 8 of a slab of
// sixteen for the heads of columns 2 t and 2 t + 1, their running maximum (the same in all g) and its share of their sums, and their
// accumulators for the channels of chunk g.  WIDE: eight heads; else at most four.
template <int D, int TS, bool WIDE>
struct AttendKv4 {
    static constexpr int WT = TS / WARPS_PER_GROUP;        // tokens per warp: 8, 16 or 32
    static constexpr int SLABS = WT > 16 ? WT / 16 : 1;
    static constexpr bool HALF = WT == 8;                  // rows 8 .. 15 of the slab do not exist
    static constexpr int MT = D / 16;                      // MMAs of a slab's first product; channel tiles of the second
    static constexpr int KW = D / 32;                      // words of a K row that a lane reads: D / 4 channels
    static constexpr int VW = D / 64;                      // words of a V row: D / 8 channels
    static constexpr Kv4Block AT = Kv4Block(TS, D);
    static constexpr float BASE = 13.f, SLACK = 1.3f;      // 2^13, e^1.3 < 2^2
    int g, t, qh, rb;
    bool head;                                             // the lane's query column is a head
    int c0;                                                // head of column 2 t (of 2 t + 1: c0 + 1)
    bool has0, has1;
    uint32_t qb[2 * MT];
    float back0, back1;                                    // undo the queries' powers of two
    float te0, te1;
    float o[MT][4], m0, m1, l0, l1;

    __device__ __forceinline__ AttendKv4(int lane, int warp, int G) {
        g = lane >> 2; t = lane & 3;
        qh = WIDE ? g : g & 3;
        head = qh < G;
        c0 = WIDE ? 2 * t : (2 * t) & 3;
        has0 = c0 < G; has1 = c0 + 1 < G;
        rb = warp * WT;
        te0 = te1 = 0.f;
        back0 = back1 = 1.f;
        reset();
    }
    __device__ __forceinline__ void reset() {
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[mt][c] = 0.f;
    }
    // q: the query of head qh (any valid row where the lane's column is no head).  Lane t of a column holds channels (D / 4) t ..
    __device__ __forceinline__ void load_q(const __nv_bfloat16* q) {
        uint32_t w[2 * MT];
#pragma unroll
        for (int k = 0; k < MT / 2; ++k) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (head) v = __ldcg(reinterpret_cast<const uint4*>(q + (D / 4) * t) + k);
            w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
        }
        uint32_t top = 0;                                  // largest magnitude, as bits
#pragma unroll
        for (int k = 0; k < 2 * MT; ++k) top = max(top, max((w[k] & 0x7fffu) << 16, w[k] & 0x7fff0000u));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int k2 = min(140 - (int)(top >> 23), 126);    // the largest lies in [2^13, 2^14) after 2^k2 (-115 .. 126)
        const float f = __uint_as_float((uint32_t)(127 + k2) << 23), back = __uint_as_float((uint32_t)(127 - k2) << 23);
#pragma unroll
        for (int k = 0; k < 2 * MT; ++k) qb[k] = pack_f16(bf16_lo(w[k]) * f, bf16_hi(w[k]) * f);
        back0 = __shfl_sync(0xffffffffu, back, 8 * t);
        back1 = __shfl_sync(0xffffffffu, back, 8 * t + 4);
    }
    // tau: the thresholds of the group's heads
    __device__ __forceinline__ void load_te(const float* tau) {
        te0 = has0 ? __ldcg(tau + c0) : 0.f;
        te1 = has1 ? __ldcg(tau + c0 + 1) : 0.f;
    }
    // the warp's maxima and sums, for a flush: m, l [8]
    __device__ __forceinline__ void store_ml(float* m, float* l) const {
        float a = l0, b = l1;
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, x);
            b += __shfl_xor_sync(0xffffffffu, b, x);
        }
        // A NaN among the weights is in all accumulators of its head by now.  They carry it on: the merge reads a sum that is not
        // above zero as no part at all.
        const bool na = a != a, nb = b != b;
        if (g == 0 && (WIDE || t < 2)) {
            m[c0] = na && m0 == -INFINITY ? 0.f : m0; m[c0 + 1] = nb && m1 == -INFINITY ? 0.f : m1;
            l[c0] = na ? 1.f : a; l[c0 + 1] = nb ? 1.f : b;
        }
    }
    // the accumulators of heads h0 .. h0 + n - 1 to sm [n][D]
    __device__ __forceinline__ void store_o(float* sm, int h0, int n) const {
        const int ha = c0 - h0, hb = ha + 1;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float x[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[c] = o[mt][c];
                if (!WIDE) x[c] += __shfl_xor_sync(0xffffffffu, x[c], 2);       // the remainders' columns
            }
            const int dcol = (D / 8) * g + 2 * mt;
            if (!WIDE && t >= 2) continue;
            if (ha >= 0 && ha < n) *reinterpret_cast<float2*>(sm + ha * D + dcol) = make_float2(x[0], x[2]);
            if (hb >= 0 && hb < n) *reinterpret_cast<float2*>(sm + hb * D + dcol) = make_float2(x[1], x[3]);
        }
    }
    __device__ __forceinline__ float gated(float S, float te, float beta, bool raw) const {
        constexpr float LOG2E = 1.4426950408889634f;
        if (te == -INFINITY || raw) return S;              // the gate is off; or the query's own token (Eq. mult_attn, s = t)
        const float x = (beta == 0.f) ? 0.f : beta * (S - te);
        return S * rcp_approx(1.f + exp2f(-x * LOG2E));    // S * sigmoid(x); exp2(+inf) -> rcp -> 0
    }
    // The block at kbase: nvalid tokens of it are in the sequence, the heads of hmask attend it, token urow (0xff: none) keeps its
    // raw logit.  release() is called when the warp has read all of the block.
    template <typename Release>
    __device__ __forceinline__ void tile(uint32_t kbase, int hmask, int urow, int nvalid, float scale, float beta, Release release) {
        constexpr float LOG2E = 1.4426950408889634f;
        const bool on0 = has0 && ((hmask >> c0) & 1), on1 = has1 && ((hmask >> (c0 + 1)) & 1);
        const float f0 = scale * back0, f1 = scale * back1;
#pragma unroll
        for (int sl = 0; sl < SLABS; ++sl) {
            const int r0 = rb + 16 * sl;
            // ---- S = K q^T
            float s[4] = {0.f, 0.f, 0.f, 0.f};
            {
                uint32_t kw[2][KW], ks[2][VW];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (HALF && h) break;
                    const int row = r0 + g + 8 * h;
                    if constexpr (D == 128) {
                        const uint4 v = lds128(kbase + row * 64 + t * 16);
                        kw[h][0] = v.x; kw[h][1] = v.y; kw[h][2] = v.z; kw[h][3] = v.w;
                        const uint32_t e = e4m3x2_to_f16x2(lds16(kbase + AT.k_scales + row * 8 + t * 2));
                        ks[h][0] = __byte_perm(e, e, 0x1010); ks[h][1] = __byte_perm(e, e, 0x3232);
                    } else {
                        const uint2 v = lds64(kbase + row * 32 + t * 8);
                        kw[h][0] = v.x; kw[h][1] = v.y;
                        ks[h][0] = e4m3x2_to_f16x2(lds8(kbase + AT.k_scales + row * 4 + t) * 0x101u);
                    }
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    uint32_t a[2][2] = {{0u, 0u}, {0u, 0u}};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (HALF && h) break;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int pair = 2 * mt + c;
                            a[h][c] = hmul2_u(e2m1x2_to_f16x2((kw[h][pair / 4] >> (8 * (pair % 4))) & 0xffu), ks[h][pair / 8]);
                        }
                    }
                    mma_f16_16816(s, a[0][0], a[1][0], a[0][1], a[1][1], qb[2 * mt], qb[2 * mt + 1]);
                }
            }
            // V's pieces are requested now so that their latency hides behind the softmax arithmetic: rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9
            uint32_t vw[4][VW], vs = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (HALF && k >= 2) break;
                const int row = r0 + 2 * t + (k & 1) + 8 * (k >> 1);
                const uint32_t base = kbase + AT.v_codes;
                if constexpr (D == 128) {
                    const uint2 v = lds64(base + row * 64 + g * 8);
                    vw[k][0] = v.x; vw[k][1] = v.y;
                    vs |= lds8(kbase + AT.v_scales + row * 8 + g) << (8 * k);
                } else {
                    vw[k][0] = lds32(base + row * 32 + g * 4);
                    vs |= lds8(kbase + AT.v_scales + row * 4 + (g >> 1)) << (8 * k);
                }
                // rows past the end of the sequence hold whatever the cache holds: keep them out of the product
                if (row >= nvalid) {
#pragma unroll
                    for (int w = 0; w < VW; ++w) vw[k][w] = 0u;
                    vs &= ~(0xffu << (8 * k));
                }
            }
            if (sl == SLABS - 1) {
                // every shared-memory read of the block has been issued before this point
                __syncwarp();
                release();
            }
            // ---- gate, mask, online softmax: tokens r0 + g and r0 + g + 8
            const int ta = r0 + g, tb = ta + 8;
            float x[4] = {gated(s[0] * f0, te0, beta, ta == urow), gated(s[1] * f1, te1, beta, ta == urow),
                          gated(s[2] * f0, te0, beta, tb == urow), gated(s[3] * f1, te1, beta, tb == urow)};
            const bool la = ta < nvalid, lb = !HALF && tb < nvalid;
            x[0] = on0 && la ? x[0] : -INFINITY;
            x[1] = on1 && la ? x[1] : -INFINITY;
            x[2] = on0 && lb ? x[2] : -INFINITY;
            x[3] = on1 && lb ? x[3] : -INFINITY;
            float b0 = fmaxf(x[0], x[2]), b1 = fmaxf(x[1], x[3]);
            if (__any_sync(0xffffffffu, b0 > m0 + SLACK || b1 > m1 + SLACK)) {
#pragma unroll
                for (int k = 4; k < 32; k <<= 1) {
                    b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, k));
                    b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, k));
                }
                const float n0 = fmaxf(m0, b0), n1 = fmaxf(m1, b1);
                const float a0 = n0 == m0 ? 1.f : exp2f((m0 - n0) * LOG2E), a1 = n1 == m1 ? 1.f : exp2f((m1 - n1) * LOG2E);   // from -inf: 0
                m0 = n0; m1 = n1;
                l0 *= a0; l1 *= a1;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) { o[mt][0] *= a0; o[mt][1] *= a1; o[mt][2] *= a0; o[mt][3] *= a1; }
            }
            const float u0 = m0 == -INFINITY ? 0.f : m0, u1 = m1 == -INFINITY ? 0.f : m1;
            float p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k] = exp2f(fmaf(x[k] - ((k & 1) ? u1 : u0), LOG2E, BASE));      // -inf gives 0
            l0 += p[0] + p[2];
            l1 += p[1] + p[3];
            // ---- P as the B operand: value and remainder
            uint32_t bh[2] = {0u, 0u}, bl[2] = {0u, 0u};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (HALF && h) break;
                const uint32_t hi = pack_f16(p[2 * h], p[2 * h + 1]);
                const uint32_t lo = pack_f16(p[2 * h] - f16_lo(hi), p[2 * h + 1] - f16_hi(hi));
                bh[h] = transpose8(WIDE || t < 2 ? hi : lo);
                if (WIDE) bl[h] = transpose8(lo);
            }
            // ---- O^T += V^T P.  A token's NaN (its scale's code) times the weight 0 of a head that does not attend the block must not
            // reach that head: where a block that some head leaves out holds one, those heads' accumulators stay as they were.
            const uint32_t s01 = e4m3x2_to_f16x2(vs & 0xffffu), s23 = HALF ? 0u : e4m3x2_to_f16x2(vs >> 16);
            const bool nan = __vcmpeq4(vs & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
            const bool keep = __any_sync(0xffffffffu, nan && !(on0 && on1));
            auto product = [&](float (&acc)[MT][4]) {
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    // bytes of (row 2 t, row 2 t + 1) codes: even channels, odd channels
                    const uint32_t e01 = (vw[0][w] & 0x0f0f0f0fu) | ((vw[1][w] & 0x0f0f0f0fu) << 4);
                    const uint32_t d01 = ((vw[0][w] >> 4) & 0x0f0f0f0fu) | (vw[1][w] & 0xf0f0f0f0u);
                    uint32_t e23 = 0, d23 = 0;
                    if (!HALF) {
                        e23 = (vw[2][w] & 0x0f0f0f0fu) | ((vw[3][w] & 0x0f0f0f0fu) << 4);
                        d23 = ((vw[2][w] >> 4) & 0x0f0f0f0fu) | (vw[3][w] & 0xf0f0f0f0u);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t a0 = hmul2_u(e2m1x2_to_f16x2((e01 >> (8 * k)) & 0xffu), s01);
                        const uint32_t a1 = hmul2_u(e2m1x2_to_f16x2((d01 >> (8 * k)) & 0xffu), s01);
                        uint32_t a2 = 0, a3 = 0;
                        if (!HALF) {
                            a2 = hmul2_u(e2m1x2_to_f16x2((e23 >> (8 * k)) & 0xffu), s23);
                            a3 = hmul2_u(e2m1x2_to_f16x2((d23 >> (8 * k)) & 0xffu), s23);
                        }
                        mma_f16_16816(acc[4 * w + k], a0, a1, a2, a3, bh[0], bh[1]);
                        if (WIDE) mma_f16_16816(acc[4 * w + k], a0, a1, a2, a3, bl[0], bl[1]);
                    }
                }
            };
            if (!keep) {
                product(o);
            } else {
                float was[MT][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) was[mt][c] = o[mt][c];
                product(o);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (!((c & 1) ? on1 : on0)) o[mt][c] = was[mt][c];
            }
        }
    }
};

}  // namespace eta
