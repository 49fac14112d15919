// Gated attention of one KV head's query heads over blocks of a 4-bit cache in shared memory, sixteen tokens (a slab) at a time: what Attend
// (eta_attend.cuh) is for bf16 tiles, with the same gate, masks and statistics.
//
// A quarter of the bytes per token leaves a quarter of the time per token, so the work per token is what has to be small:
//   - tokens are the rows of the first product (S = K q^T: sixteen tokens an MMA, query heads its eight columns), channels the rows of the second
//     (O^T = V^T P), so that no row of an MMA is padding; the probabilities get from one's layout to the other's by a transpose of 8x8.
//   - a code is converted by the hardware, two at a time, and scaled as an fp16 pair: code * scale is exact in fp16, so both products are
//     exact and their sums fp32.  Queries are scaled by a power of two per head to use fp16's range: bf16's eight bits stay whole down to
//     2^-30 of the head's largest channel, below that fewer of them, and nothing under 2^-38.
//   - probabilities are fed as the nearest fp16 value and 2^11 times what that leaves, in fp16 (24 bits; remainders as they are would be subnormal from
//     2^-12 of the largest weight on, and all that an output is made of is smaller where one token has the weight and next to no value).  Up
//     to four heads, both are columns of one MMA: columns 4 to 7 repeat the heads of 0 to 3, whose lanes compute the same scores again and feed
//     the remainder.  With eight heads the remainders' MMA starts from zero and its sums are added 2^-11 fold.
//   - the running maximum follows the scores only when one is more than SLACK above it: exp(s - m) is then at most 2^6, and with
//     the factor 2^BASE, which every part carries and the final division drops, inside fp16's range at both ends.
// Where every block is attended, what bounds it is the scheduler: a conversion makes two numbers in two cycles of one, an MMA takes eight that add to
// them.  16 x 8K to 64K tokens, 4 KV heads of eight: 97 to 99 us a step (340 MB: 3.4 TB/s, half a copy's rate; 57 M warp instructions in 56 % of the
// streaming kernel's issue slots, 22 M of them on the ALU pipe).  4 x 128K of 8 KV heads, a tenth of the blocks: 35 us, where
// the streaming kernel's instructions fill 44 % of its issue slots and its warps wait for memory most; neither bytes nor instructions bound it.
#pragma once

#include <float.h>

#include "eta_attend.cuh"
#include "eta_kv4.cuh"

namespace eta {

// shared-memory loads at a constant distance from an address
template <int AT> __device__ __forceinline__ uint4 lds128_at(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4+%5];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint2 lds64_at(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2+%3];" : "=r"(v.x), "=r"(v.y) : "r"(addr), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint32_t lds32_at(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1+%2];" : "=r"(v) : "r"(addr), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint32_t lds16_at(uint32_t addr) {
    uint32_t v;
    asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1+%2];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v) : "r"(addr), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint32_t lds8_at(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1+%2];" : "=r"(v) : "r"(addr), "n"(AT));
    return v;
}
// D = A B: the first MMA of a chain
__device__ __forceinline__ void mma_f16_16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// 8x8 matrix of 16-bit elements, two neighbours of a row per lane: transposed
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// a, b -= 2048 times the halves of v: exact
__device__ __forceinline__ void sub_rest(float& a, float& b, uint32_t v) {
    asm("{\n\t.reg .b16 l, h, m;\n\tmov.b32 {l, h}, %2;\n\tmov.b16 m, 0xe800;\n\t"
        "fma.rn.f32.f16 %0, l, m, %0;\n\tfma.rn.f32.f16 %1, h, m, %1;\n\t}"
        : "+f"(a), "+f"(b) : "r"(v));
}

__device__ __forceinline__ bool has_nan(uint32_t p) {
    const __half2 h = *reinterpret_cast<const __half2*>(&p);
    return !__hbeq2(h, h);
}
__device__ __forceinline__ uint32_t without_nan(uint32_t p) {      // a NaN as zero
    if ((p & 0x7fffu) > 0x7c00u) p &= 0xffff0000u;
    if ((p & 0x7fff0000u) > 0x7c000000u) p &= 0xffffu;
    return p;
}

// One warp's part.  Lane (g, t) = (lane / 4, lane % 4) holds the scores of tokens g and g + 8 of a slab for the heads of columns 2 t and 2 t + 1,
// their running maximum (the same in all g) and its share of their sums, and their accumulators for the channels of chunk g.
// b: tokens of a block.  WIDE: eight heads; else at most four.
template <int D, int b, bool WIDE>
struct AttendKv4 {
    static constexpr int MT = D / 16;                      // MMAs of a slab's first product; channel tiles of the second
    static constexpr int KW = D / 32;                      // words of a K row that a lane reads: D / 4 channels
    static constexpr int VW = D / 64;                      // words of a V row: D / 8 channels
    static constexpr int CR = D / 2, SR = D / 16;          // bytes of a row's codes and scales
    static constexpr Kv4Block AT = Kv4Block(b, D);
    static constexpr float BASE = 9.f, SLACK = 4.f;        // 2^9, e^4 < 2^6
    static constexpr float REST = 2048.f;                  // what remainders are multiplied with
    static constexpr float NONE = -FLT_MAX;                // the maximum of no score: every other number is more than SLACK above it
    int g, t, qh;
    bool head;                                             // the lane's query column is a head
    int c0;                                                // head of column 2 t (of 2 t + 1: c0 + 1)
    bool has0, has1;
    uint32_t all;                                          // bits of the group's heads
    bool rest;                                             // up to four heads: the lane feeds a weight's remainder, not the value
    uint32_t qb[2 * MT];
    float back0, back1;                                    // undo the queries' powers of two
    float te0, te1;
    bool gate_on;                                          // some head of the row has a threshold: the same for the whole warp
    float o[MT][4], m0, m1, l0, l1;
    // where the lane's pieces of a slab begin: K codes and scales (row g), V codes and scales (row 2 t)
    uint32_t kc, ks, vc, vs;

    __device__ __forceinline__ AttendKv4(int lane, int, int G) {
        g = lane >> 2; t = lane & 3;
        qh = WIDE ? g : g & 3;
        head = qh < G;
        c0 = WIDE ? 2 * t : (2 * t) & 3;
        has0 = c0 < G; has1 = c0 + 1 < G;
        all = (1u << G) - 1;
        rest = t >= 2;
        te0 = te1 = 0.f;
        gate_on = true;
        back0 = back1 = 1.f;
        kc = g * CR + t * (D / 8);
        ks = AT.k_scales + g * SR + t * (D / 64);
        vc = AT.v_codes + 2 * t * CR + g * (D / 16);
        vs = AT.v_scales + 2 * t * SR + (D == 128 ? g : g >> 1);
        reset();
    }
    __device__ __forceinline__ void reset() {
        m0 = m1 = k0 = k1 = NONE;
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
        te0 = has0 ? __ldcg(tau + c0) : -INFINITY;
        te1 = has1 ? __ldcg(tau + c0 + 1) : -INFINITY;
        gate_on = __any_sync(0xffffffffu, te0 != -INFINITY || te1 != -INFINITY);
    }
    // the warp's maxima and sums, for a flush: m, l [8]
    __device__ __forceinline__ void store_ml(float* m, float* l) const {
        float x = l0, y = l1;
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) {
            x += __shfl_xor_sync(0xffffffffu, x, k);
            y += __shfl_xor_sync(0xffffffffu, y, k);
        }
        // A NaN among the weights is in all accumulators of its head by now.  They carry it on: the merge reads a sum that is not
        // above zero as no part at all.
        const bool nx = x != x, ny = y != y;
        if (g == 0 && (WIDE || t < 2)) {
            m[c0] = m0 != NONE ? m0 : (nx ? 0.f : -INFINITY); m[c0 + 1] = m1 != NONE ? m1 : (ny ? 0.f : -INFINITY);
            l[c0] = nx ? 1.f : x; l[c0 + 1] = ny ? 1.f : y;
        }
    }
    // The warp's accumulators are folded into sm [heads][O_STRIDE] every FOLD stages and at the end of a piece: an MMA cuts its sum off where
    // fp32 would round it, and after two hundred of them in a row (64K tokens, dense) an output was off by
    // 1.9e-6 of itself, by 7e-7 with the sums folded; with remainders fed REST fold as well it is 3.5e-7.
    // Channel (D / 8) g + 2 mt + c is at 16 mt + 2 g + c: the sixteen lanes of a phase meet every bank once.
    static constexpr int O_STRIDE = D + 4, FOLD = 10;
    // where four consecutive channels 4 k .. are: two pairs, 16 floats apart
    __device__ __forceinline__ static int o_at(int k) { return 16 * (2 * k % MT) + 2 * (2 * k / MT); }
    float k0, k1;                                          // the maxima that sm's sums go with
    template <bool FIRST>
    __device__ __forceinline__ void fold(float* sm) {
        constexpr float LOG2E = 1.4426950408889634f;
        const float f0 = FIRST ? 0.f : ex2_approx((k0 - m0) * LOG2E), f1 = FIRST ? 0.f : ex2_approx((k1 - m1) * LOG2E);   // (from NONE: 0)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float x[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[c] = o[mt][c];
                if (!WIDE) x[c] = fmaf(__shfl_xor_sync(0xffffffffu, x[c], 2), 1.f / REST, x[c]);       // values' columns and remainders'
                o[mt][c] = 0.f;
            }
            if (!WIDE && t >= 2) continue;
            float2* const pa = reinterpret_cast<float2*>(sm + c0 * O_STRIDE + 16 * mt + 2 * g);
            float2* const pb = pa + O_STRIDE / 2;
            if (has0) {
                if (FIRST) *pa = make_float2(x[0], x[2]);
                else *pa = make_float2(fmaf(pa->x, f0, x[0]), fmaf(pa->y, f0, x[2]));
            }
            if (has1) {
                if (FIRST) *pb = make_float2(x[1], x[3]);
                else *pb = make_float2(fmaf(pb->x, f1, x[1]), fmaf(pb->y, f1, x[3]));
            }
        }
        k0 = m0; k1 = m1;
    }
    __device__ __forceinline__ float gated(float S, float te, float beta) const {
        constexpr float LOG2E = 1.4426950408889634f;
        const float x = (beta == 0.f) ? 0.f : beta * (S - te);
        const float y = S * rcp_approx(1.f + ex2_approx(-x * LOG2E));    // S * sigmoid(x); 2^inf -> rcp -> 0
        return te == -INFINITY ? S : y;
    }
    // The slab of tokens r0 .. r0 + 15 of the block at blk: nvalid tokens of the block are in the sequence, the heads of hmask attend
    // it, token urow (0xff: none) keeps its raw logit.
    __device__ __forceinline__ void slab(uint32_t blk, int r0, int hmask, int urow, int nvalid, float scale, float beta) {
        constexpr float LOG2E = 1.4426950408889634f;
        // ---- S = K q^T: rows r0 + g and r0 + g + 8
        float s[4];
        const uint32_t kca = blk + kc + r0 * CR, ksa = blk + ks + r0 * SR, vca = blk + vc + r0 * CR, vsa = blk + vs + r0 * SR;
        {
            uint32_t kf[2][KW][4], sc[2][VW];
            if constexpr (D == 128) {
                const uint4 x = lds128_at<0>(kca), y = lds128_at<8 * CR>(kca);
                const uint32_t e = e4m3x2_to_f16x2(lds16_at<0>(ksa)), f = e4m3x2_to_f16x2(lds16_at<8 * SR>(ksa));
                e2m1x8_to_f16x2(x.x, kf[0][0]); e2m1x8_to_f16x2(x.y, kf[0][1]); e2m1x8_to_f16x2(x.z, kf[0][2]); e2m1x8_to_f16x2(x.w, kf[0][3]);
                e2m1x8_to_f16x2(y.x, kf[1][0]); e2m1x8_to_f16x2(y.y, kf[1][1]); e2m1x8_to_f16x2(y.z, kf[1][2]); e2m1x8_to_f16x2(y.w, kf[1][3]);
                sc[0][0] = __byte_perm(e, e, 0x1010); sc[0][1] = __byte_perm(e, e, 0x3232);
                sc[1][0] = __byte_perm(f, f, 0x1010); sc[1][1] = __byte_perm(f, f, 0x3232);
            } else {
                const uint2 x = lds64_at<0>(kca), y = lds64_at<8 * CR>(kca);
                e2m1x8_to_f16x2(x.x, kf[0][0]); e2m1x8_to_f16x2(x.y, kf[0][1]);
                e2m1x8_to_f16x2(y.x, kf[1][0]); e2m1x8_to_f16x2(y.y, kf[1][1]);
                sc[0][0] = e4m3x2_to_f16x2(lds8_at<0>(ksa) * 0x101u);
                sc[1][0] = e4m3x2_to_f16x2(lds8_at<8 * SR>(ksa) * 0x101u);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int w = mt / 2, k = 2 * (mt % 2);
                const uint32_t a0 = hmul2_u(kf[0][w][k], sc[0][mt / 4]), a1 = hmul2_u(kf[1][w][k], sc[1][mt / 4]);
                const uint32_t a2 = hmul2_u(kf[0][w][k + 1], sc[0][mt / 4]), a3 = hmul2_u(kf[1][w][k + 1], sc[1][mt / 4]);
                if (mt == 0) mma_f16_16816_first(s, a0, a1, a2, a3, qb[0], qb[1]);
                else mma_f16_16816(s, a0, a1, a2, a3, qb[2 * mt], qb[2 * mt + 1]);
            }
        }
        // V's pieces are requested now so that their latency hides behind the softmax arithmetic: rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        uint32_t vw[4][VW], s01, s23;
        {
            if constexpr (D == 128) {
                const uint2 x0 = lds64_at<0>(vca), x1 = lds64_at<CR>(vca), x2 = lds64_at<8 * CR>(vca), x3 = lds64_at<9 * CR>(vca);
                vw[0][0] = x0.x; vw[0][1] = x0.y; vw[1][0] = x1.x; vw[1][1] = x1.y;
                vw[2][0] = x2.x; vw[2][1] = x2.y; vw[3][0] = x3.x; vw[3][1] = x3.y;
            } else {
                vw[0][0] = lds32_at<0>(vca); vw[1][0] = lds32_at<CR>(vca); vw[2][0] = lds32_at<8 * CR>(vca); vw[3][0] = lds32_at<9 * CR>(vca);
            }
            uint32_t e01 = __byte_perm(lds8_at<0>(vsa), lds8_at<SR>(vsa), 0x5540), e23 = __byte_perm(lds8_at<8 * SR>(vsa), lds8_at<9 * SR>(vsa), 0x5540);
            if (nvalid < r0 + 16) {
                // rows past the end of the sequence hold whatever the cache holds: keep them out of the product
                const int n = nvalid - r0 - 2 * t;         // of rows 0, 1, 8, 9 from the lane's first those below n are in the sequence
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    if (n < 1) vw[0][w] = 0u;
                    if (n < 2) vw[1][w] = 0u;
                    if (n < 9) vw[2][w] = 0u;
                    if (n < 10) vw[3][w] = 0u;
                }
                if (n < 1) e01 &= 0xff00u;
                if (n < 2) e01 &= 0x00ffu;
                if (n < 9) e23 &= 0xff00u;
                if (n < 10) e23 &= 0x00ffu;
            }
            s01 = e4m3x2_to_f16x2(e01);
            s23 = e4m3x2_to_f16x2(e23);
        }
        // ---- gate, mask, online softmax
        const float f0 = scale * back0, f1 = scale * back1;
        float x[4] = {s[0] * f0, s[1] * f1, s[2] * f0, s[3] * f1};
        if (gate_on) {
            const float raw[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = gated(raw[k], (k & 1) ? te1 : te0, beta);
            if (urow != 0xff) {                            // the query's own token (Eq. mult_attn, s = t)
                if (r0 + g == urow) { x[0] = raw[0]; x[1] = raw[1]; }
                if (r0 + g + 8 == urow) { x[2] = raw[2]; x[3] = raw[3]; }
            }
        }
        if ((~hmask & all) != 0 || nvalid < r0 + 16) {     // some head leaves the block out, or some row is past the end
            const bool on0 = has0 && ((hmask >> c0) & 1), on1 = has1 && ((hmask >> (c0 + 1)) & 1);
            const bool la = r0 + g < nvalid, lb = r0 + g + 8 < nvalid;
            x[0] = on0 && la ? x[0] : -INFINITY;
            x[1] = on1 && la ? x[1] : -INFINITY;
            x[2] = on0 && lb ? x[2] : -INFINITY;
            x[3] = on1 && lb ? x[3] : -INFINITY;
            if (__any_sync(0xffffffffu, has_nan(s01) || has_nan(s23))) {
                // A NaN in V, which is a scale's, must not reach the heads that leave the block out, as 0 * NaN would.  The scale is taken as
                // zero, and the heads that attend the block get their NaN in the group's channels, which are the chunk of the lanes of one g.
                const unsigned lanes = __ballot_sync(0xffffffffu, has_nan(s01) || has_nan(s23));
                s01 = without_nan(s01); s23 = without_nan(s23);
                if (lanes & ((D == 128 ? 0xfu : 0xffu) << (4 * (D == 128 ? g : g & ~1)))) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if ((c & 1) ? on1 : on0) o[mt][c] = __uint_as_float(0x7fffffffu);
                }
            }
        }
        float b0 = fmaxf(x[0], x[2]), b1 = fmaxf(x[1], x[3]);
        if (__any_sync(0xffffffffu, b0 - m0 > SLACK || b1 - m1 > SLACK)) {       // (the differences are exact where it matters)
#pragma unroll
            for (int k = 4; k < 32; k <<= 1) {
                b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, k));
                b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, k));
            }
            const float n0 = fmaxf(m0, b0), n1 = fmaxf(m1, b1);
            const float a0 = ex2_approx((m0 - n0) * LOG2E), a1 = ex2_approx((m1 - n1) * LOG2E);       // from NONE: 0
            m0 = n0; m1 = n1;
            l0 *= a0; l1 *= a1;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) { o[mt][0] *= a0; o[mt][1] *= a1; o[mt][2] *= a0; o[mt][3] *= a1; }
        }
        float p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = ex2_approx(fmaf(x[k] - ((k & 1) ? m1 : m0), LOG2E, BASE));      // -inf gives 0
        l0 += p[0] + p[2];
        l1 += p[1] + p[3];
        // ---- P as the B operand: the nearest fp16 value, and REST times what that leaves.  A weight is held to 2^-24 of itself, or to 2^-36 in p, that is
        // 2^-45 of the warp's largest, where that is more.
        uint32_t bh[2], bl[2] = {0u, 0u};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t v = pack_f16(p[2 * h], p[2 * h + 1]);
            float r0, r1;
            mul2(r0, r1, p[2 * h], p[2 * h + 1], REST, REST);
            sub_rest(r0, r1, v);
            const uint32_t r = pack_f16(r0, r1);
            bh[h] = transpose8(WIDE ? v : (rest ? r : v));
            if (WIDE) bl[h] = transpose8(r);
        }
        // ---- O^T += V^T P
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            // bytes of (row 2 t, row 2 t + 1) codes: even channels, odd channels
            uint32_t e01[4], d01[4], e23[4], d23[4];
            e2m1x8_to_f16x2((vw[0][w] & 0x0f0f0f0fu) | ((vw[1][w] * 16u) & 0xf0f0f0f0u), e01);
            e2m1x8_to_f16x2(((vw[0][w] >> 4) & 0x0f0f0f0fu) | (vw[1][w] & 0xf0f0f0f0u), d01);
            e2m1x8_to_f16x2((vw[2][w] & 0x0f0f0f0fu) | ((vw[3][w] * 16u) & 0xf0f0f0f0u), e23);
            e2m1x8_to_f16x2(((vw[2][w] >> 4) & 0x0f0f0f0fu) | (vw[3][w] & 0xf0f0f0f0u), d23);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                e01[k] = hmul2_u(e01[k], s01); d01[k] = hmul2_u(d01[k], s01); e23[k] = hmul2_u(e23[k], s23); d23[k] = hmul2_u(d23[k], s23);
                mma_f16_16816(o[4 * w + k], e01[k], d01[k], e23[k], d23[k], bh[0], bh[1]);
            }
            if (WIDE) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x[4];
                    mma_f16_16816_first(x, e01[k], d01[k], e23[k], d23[k], bl[0], bl[1]);
                    fma2(o[4 * w + k][0], o[4 * w + k][1], x[0], x[1], 1.f / REST, 1.f / REST);
                    fma2(o[4 * w + k][2], o[4 * w + k][3], x[2], x[3], 1.f / REST, 1.f / REST);
                }
            }
        }
    }
};

}  // namespace eta
