// Block summaries (Section 3) of a 4-bit cache: centroid, coordinate-wise population deviation and largest norm of the keys as they
// are stored, at prefill for all blocks and at a decode step for the block that the newest token completed.
//
// One warp owns one block of b keys.  A lane holds one group of sixteen channels, which share a scale: 8 bytes of codes and a scale
// byte a row, 32 / (d / 16) rows per warp instruction.  A key's coordinate is code * scale, an exact fp16 number of at most six
// significant bits; its square has twelve, so that the sums of 32 to 128 of either are exact in fp32, or as good as: the deviation
// comes from the plain moments,
//   mu = S1 / b,   sigma^2 = S2 / b - mu^2   (one fma),
// without the shift that bf16 keys need, and is exactly 0 for identical keys.  A row's squared norm is summed group by group from
// the codes' squares (quarters, up to 288 in either half of an fp16 pair: exact) times the scale's square.
// Build and append run the same routine: appending a block gives the bytes rebuilding it would.
// 4 x 128K tokens of 8 heads take 127 to 129 us (336 MB: 2.6 TB/s, 40 % of a copy's rate): 104 M warp instructions, 65 M of them the moments' on the FMA
// pipe, fill 72 % of the issue slots.  The rest is the wait for the next eight rows, which are asked for only when the last eight are summed.
#include "eta_kv4.cuh"

namespace eta {

// Sixteen codes of a lane as fp16 pairs, unscaled
__device__ __forceinline__ void codes_to_f16(const uint2& w, uint32_t (&h)[8]) {
    uint32_t x[4], y[4];
    e2m1x8_to_f16x2(w.x, x);
    e2m1x8_to_f16x2(w.y, y);
#pragma unroll
    for (int k = 0; k < 4; ++k) { h[k] = x[k]; h[4 + k] = y[k]; }
}
// a, b += the two halves of v;  c, d += their squares.  sm_100 adds and multiplies fp16 numbers into fp32 ones: unpacking them first cost half of the
// pass (155 -> 129 us for 4 x 128K tokens of 8 heads).
__device__ __forceinline__ void add_moments(float& a, float& b, float& c, float& d, uint32_t v) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %4;\n\t"
        "add.rn.f32.f16 %0, l, %0;\n\tadd.rn.f32.f16 %1, h, %1;\n\t"
        "fma.rn.f32.f16 %2, l, l, %2;\n\tfma.rn.f32.f16 %3, h, h, %3;\n\t}"
        : "+f"(a), "+f"(b), "+f"(c), "+f"(d) : "r"(v));
}

template <int D, bool ENVELOPE>
__device__ __forceinline__ void summarize_kv4(const unsigned char* blk, int b, float g, unsigned char* rec, bool packed, float* mn) {
    constexpr int LPR = D / KV4_GROUP;        // lanes per row
    constexpr int RPP = 32 / LPR;             // rows per pass
    constexpr int U = D == 128 ? 8 : 4;       // passes in flight; b is a multiple of U * RPP
    constexpr int CH = KV4_GROUP / RPP;       // channels whose sums a lane ends up with
    const int lane = threadIdx.x & 31, cc = lane % LPR, ro = lane / LPR;
    const unsigned char* codes = blk + ro * (D / 2) + cc * 8;
    const unsigned char* scales = blk + Kv4Block(b, D).k_scales + ro * LPR + cc;
    float s1[KV4_GROUP], s2[KV4_GROUP], n2[U], maxn2 = 0.f;
#pragma unroll
    for (int k = 0; k < KV4_GROUP; ++k) { s1[k] = 0.f; s2[k] = 0.f; }
    for (int t0 = 0; t0 < b; t0 += U * RPP) {
        uint2 w[U];
        uint32_t sc[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            w[u] = __ldcg(reinterpret_cast<const uint2*>(codes + (t0 + u * RPP) * (D / 2)));
            sc[u] = __ldcg(scales + (t0 + u * RPP) * LPR);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t h[8];
            codes_to_f16(w[u], h);
            const uint32_t s = e4m3x2_to_f16x2(sc[u] * 0x101u);
            uint32_t sq = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sq = hfma2_u(h[k], h[k], sq);
                add_moments(s1[2 * k], s1[2 * k + 1], s2[2 * k], s2[2 * k + 1], hmul2_u(h[k], s));
            }
            const float sf = f16_lo(s);
            n2[u] = (f16_lo(sq) + f16_hi(sq)) * (sf * sf);
        }
        // the rows' lanes meet: every exchange halves the rows that a lane goes on with
#pragma unroll
        for (int x = 1, n = U; x < LPR; x <<= 1, n >>= 1) {
            const bool up = (lane & x) != 0;
#pragma unroll
            for (int u = 0; u < n / 2; ++u) {
                const float o = up ? n2[u] : n2[n / 2 + u];
                n2[u] = (up ? n2[n / 2 + u] : n2[u]) + __shfl_xor_sync(0xffffffffu, o, x);
            }
        }
        static_assert(U == LPR, "a row for every lane of a row");
        maxn2 = max_nan(maxn2, n2[0]);
    }
#pragma unroll
    for (int x = 1; x < LPR; x <<= 1) maxn2 = max_nan(maxn2, __shfl_xor_sync(0xffffffffu, maxn2, x));
#pragma unroll
    for (int x = LPR; x < 32; x <<= 1) maxn2 = max_nan(maxn2, __shfl_xor_sync(0xffffffffu, maxn2, x));
    const float inv_b = 1.0f / (float)b;
    if (ENVELOPE) {
        // the sums of all rows in every lane, then a second pass: four tokens are four row groups
#pragma unroll
        for (int x = LPR; x < 32; x <<= 1)
#pragma unroll
            for (int k = 0; k < KV4_GROUP; ++k) s1[k] += __shfl_xor_sync(0xffffffffu, s1[k], x);
#pragma unroll
        for (int k = 0; k < KV4_GROUP; ++k) s2[k] = 0.f;
        for (int t = 0; t < b; t += RPP) {
            uint32_t h[8];
            codes_to_f16(__ldcg(reinterpret_cast<const uint2*>(codes + t * (D / 2))), h);
            const uint32_t s = e4m3x2_to_f16x2((uint32_t)__ldcg(scales + t * LPR) * 0x101u);
#pragma unroll
            for (int k = 0; k < KV4_GROUP; ++k) {
                const uint32_t v = hmul2_u(h[k / 2], s);
                const float dv = ((k & 1) ? f16_hi(v) : f16_lo(v)) - s1[k] * inv_b;
                float q = dv * dv;
                q += __shfl_xor_sync(0xffffffffu, q, LPR);
                q += __shfl_xor_sync(0xffffffffu, q, 2 * LPR);
                s2[k] = max_nan(s2[k], q);
            }
        }
#pragma unroll
        for (int k = 0; k < KV4_GROUP; ++k) {
            if (RPP == 8) s2[k] = max_nan(s2[k], __shfl_xor_sync(0xffffffffu, s2[k], 16));
            s2[k] *= 0.25f;
        }
    }
    // Row groups meet: every exchange halves the channels that a lane goes on with (the envelope's sums are whole in every lane, which only
    // selects).  c0: the lane's first channel at the end.
    int c0 = cc * KV4_GROUP;
#pragma unroll
    for (int x = LPR, n = KV4_GROUP; x < 32; x <<= 1, n >>= 1) {
        const bool up = (lane & x) != 0;
        if (up) c0 += n / 2;
#pragma unroll
        for (int k = 0; k < n / 2; ++k) {
            const float o1 = up ? s1[k] : s1[n / 2 + k], o2 = up ? s2[k] : s2[n / 2 + k];
            s1[k] = up ? s1[n / 2 + k] : s1[k];
            s2[k] = up ? s2[n / 2 + k] : s2[k];
            if (!ENVELOPE) {
                s1[k] += __shfl_xor_sync(0xffffffffu, o1, x);
                s2[k] += __shfl_xor_sync(0xffffffffu, o2, x);
            }
        }
    }
    float mu[CH], sg[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const float mean = s1[k] * inv_b;
        const float var = ENVELOPE ? s2[k] : max_nan(fmaf(-mean, mean, s2[k] * inv_b), 0.f);
        mu[k] = mean * g;
        sg[k] = sqrtf(var) * g;
    }
    uint32_t m16[CH / 2], s16[CH / 2], s8 = 0;
#pragma unroll
    for (int k = 0; k < CH / 2; ++k) {
        const __half2 m = __floats2half2_rn(mu[2 * k], mu[2 * k + 1]), s = __floats2half2_rn(sg[2 * k], sg[2 * k + 1]);
        m16[k] = *reinterpret_cast<const uint32_t*>(&m);
        s16[k] = *reinterpret_cast<const uint32_t*>(&s);
        if (packed) s8 |= (f32_to_e4m3_up(sg[2 * k]) | (f32_to_e4m3_up(sg[2 * k + 1]) << 8)) << (16 * k);
    }
    if constexpr (CH == 4) {
        *reinterpret_cast<uint2*>(rec + 2 * c0) = make_uint2(m16[0], m16[1]);
        if (packed) *reinterpret_cast<uint32_t*>(rec + 2 * D + c0) = s8;
        else *reinterpret_cast<uint2*>(rec + 2 * D + 2 * c0) = make_uint2(s16[0], s16[1]);
    } else {
        *reinterpret_cast<uint32_t*>(rec + 2 * c0) = m16[0];
        if (packed) *reinterpret_cast<uint16_t*>(rec + 2 * D + c0) = (uint16_t)s8;
        else *reinterpret_cast<uint32_t*>(rec + 2 * D + 2 * c0) = s16[0];
    }
    if (lane == 0) *mn = sqrtf(maxn2) * g;
}

struct Kv4IndexArgs {
    const unsigned char* pool;
    int64_t sb, sh, sj;
    float g;
    int Hkv, b, t_cap, nb_cap, nb_max, newest, mode;
    int64_t warps;
    const int32_t *seq_lens, *table;
    int table_stride;
    unsigned char* musig;
    float* mnorm;
};

// A warp per (row, block), or where only the newest blocks are asked for per row.
template <int D>
__global__ void __launch_bounds__(128) summaries_kv4_kernel(const Kv4IndexArgs a) {
    pdl_wait();
    if (a.newest) pdl_trigger();       // nothing later in a decode step needs the new record before it has waited for it
    const int64_t wid = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (wid >= a.warps) return;
    const int r = a.newest ? (int)wid : (int)(wid / a.nb_max);
    int j = (int)(wid - (int64_t)r * a.nb_max);
    const int i = r / a.Hkv, hk = r % a.Hkv;
    int T = __ldcg(a.seq_lens + i);
    if (a.newest) {
        if (T <= 0 || T > a.t_cap || T % a.b != 0) return;
        j = T / a.b - 1;
    } else {
        T = T < 0 ? 0 : (T > a.t_cap ? a.t_cap : T);
        if (j >= T / a.b) return;
    }
    if (j >= a.nb_cap) return;
    const unsigned char* blk = a.pool + hk * a.sh + (a.table ? (int64_t)__ldcg(a.table + (int64_t)i * a.table_stride + j) * a.sb
                                                             : i * a.sb + j * a.sj);
    const int64_t rec = (int64_t)r * a.nb_cap + j;
    const bool packed = (a.mode & 2) != 0;      // mode: bit 0 sub-block envelope, bit 1 packed records
    unsigned char* to = a.musig + rec * (packed ? 3 * D : 4 * D);
    if (a.mode & 1) summarize_kv4<D, true>(blk, a.b, a.g, to, packed, a.mnorm + rec);
    else summarize_kv4<D, false>(blk, a.b, a.g, to, packed, a.mnorm + rec);
}

static int summaries_kv4(const eta_cache_desc* desc, const eta_kv4_desc* kv4, const eta_page_table* pages, const void* pool,
                         const int32_t* seq_lens, void* musig, float* mnorm, uint32_t flags, bool newest, const char* what, void* stream) {
    int rc = validate_index(desc);
    if (rc != ETA_OK) return rc;
    if (pages && (rc = validate_pages(desc, pages)) != ETA_OK) return rc;
    if ((rc = validate_kv4(desc, kv4, pool, pages != nullptr)) != ETA_OK) return rc;
    if (!seq_lens || !musig || !mnorm || (flags & ~(ETA_BUILD_SIGMA_ENVELOPE | ETA_BUILD_PACKED_SIGMA))) return ETA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(musig) & 15) return ETA_ERR_UNSUPPORTED;
    Kv4IndexArgs a;
    a.pool = static_cast<const unsigned char*>(pool);
    a.sb = kv4->stride_b; a.sh = kv4->stride_h; a.sj = pages ? 0 : kv4->stride_j; a.g = kv4->k_scale;
    a.Hkv = desc->n_kv_heads; a.b = desc->block_size; a.t_cap = desc->t_cap; a.nb_cap = desc->nb_cap;
    a.nb_max = newest ? 0 : desc->t_cap / desc->block_size;
    a.newest = newest; a.mode = (int)flags;
    const int64_t rows = (int64_t)desc->batch * desc->n_kv_heads;
    a.warps = newest ? rows : rows * a.nb_max;
    if (a.warps == 0) return ETA_OK;
    if ((a.warps + 3) / 4 > INT32_MAX) return ETA_ERR_UNSUPPORTED;
    a.seq_lens = seq_lens;
    a.table = pages ? pages->block_table : nullptr;
    a.table_stride = pages ? pages->table_stride : 0;
    a.musig = static_cast<unsigned char*>(musig);
    a.mnorm = mnorm;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (newest) profile_mark(0, s);
    return launch_pdl(what, desc->head_dim == 128 ? summaries_kv4_kernel<128> : summaries_kv4_kernel<64>, dim3((unsigned)((a.warps + 3) / 4)),
                      dim3(128), 0, s, a);
}

}  // namespace eta

extern "C" {

int eta_build_block_summaries_kv4(const eta_cache_desc* desc, const eta_kv4_desc* kv4, const eta_page_table* pages, const void* pool,
                                  const int32_t* seq_lens, void* musig, float* mnorm, uint32_t flags, void* stream) {
    return eta::summaries_kv4(desc, kv4, pages, pool, seq_lens, musig, mnorm, flags, false, "eta_build_block_summaries_kv4", stream);
}

int eta_append_summary_kv4(const eta_cache_desc* desc, const eta_kv4_desc* kv4, const eta_page_table* pages, const void* pool,
                           const int32_t* seq_lens_after, void* musig, float* mnorm, uint32_t flags, void* stream) {
    return eta::summaries_kv4(desc, kv4, pages, pool, seq_lens_after, musig, mnorm, flags, true, "eta_append_summary_kv4", stream);
}

}  // extern "C"
