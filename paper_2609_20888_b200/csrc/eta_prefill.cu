// Attention of a step's new tokens over the cache that holds them already: prompts, chunks of prompts and single tokens, packed, each
// sequence behind its own context.
//
//   out[r, h] = sum_{t <= p(r)} w_t v_t / sum_{t <= p(r)} w_t,   w = exp(S~),   S = s <q_h, k_t>
//   S~ = S (softmax), or S sigmoid(beta (S - tau_eff)) (Eq. mult_attn), raw for t = p(r) with ETA_FLAG_UNGATE_LAST
//
// A work item is 256 query rows of one (sequence, KV head): 256 / G tokens with the G heads of the group packed behind each other, so
// that a tile of K and V serves them all.  The rows are two halves of 128, which take turns on the tensor core: while one half's scores
// are turned into weights the other half's products run.  An item with rows for one half only (a single token) gives them to both
// halves, which take the tiles in turns; the second hands its sums to the first at the end.
//   tensor memory   S of each half (128 fp32 columns; its weights, bf16, overwrite the first 64), O of each half (head_dim columns)
//   shared memory   the queries (two halves), a ring of K and V tiles of 128 tokens (128-byte swizzle, 64-column halves)
//   warps           0-15 softmax and epilogue, two threads to a row; 16 copies (TMA, a copy per page and 64 columns); 17 issues the MMAs;
//                   18, 19 clean tiles
// S = Q K^T has both operands in shared memory; O += P V takes P from tensor memory and V as it lies (token-major).
// The running maximum moves only when it would by more than 2^8: weights are then at most 2^8 and O is rescaled a few times a row
// instead of once a tile.  Weights are rounded to bf16 (relative 2^-8, as much as the output's own rounding); their sum, O and
// the maximum are fp32.
//
// What bounds it: a tile of a half is a chain, S -> maximum (480 to 570 cycles) -> the two threads of a row meet (200) -> weights (830 to 1000
// for each chunk, with the other half's beside them) -> O, and 500 more until the next S is there, in the clock of the softmax warps at head_dim 128;
// there is tensor memory for two halves' chains, not three.  Tensor core and special function unit have 2048 cycles of work a tile each and are
// busy 51 % of the time.  One 8K prompt of 32 / 8 heads of 128 takes 530 to 600 us, 32K 7.7 to 8.9 ms (1.0 to 1.1 PFLOP/s; by the power limit).  With parts
// taken out of a kernel two steps earlier 32K took 6.3 to 6.8 ms without the products, as much without the softmax, 3.8 without both and without copies.  Gated scores take
// one and a quarter more special functions each (60 to 69 % busy) and 980 instructions a thread and tile instead of 490: 11 packed prompts to 5K
// 1.00 ms (530 TFLOP/s; with a reciprocal for two gates instead of four 1.03), 2 x 1111 tokens behind 32K at head_dim 64 650 us (320 TFLOP/s).
// 64 single tokens behind 16K stream at 6.0 TB/s.
// Tried, for the 32K prompt: a thread per row and eight softmax warps 8.4 to 9.4 ms; a warp for each half's MMAs, free 10.3, taking turns 8.9 (the
// halves fall into step; a token for the special function unit keeps them apart and costs what it gains); a quarter of the exponentials as polynomials on the fp32
// pipe 9.2 (power); steps of 64 tokens with the next scores worked out ahead 11.9 (twice the hand-overs; an S of 64 columns runs at two
// thirds of the rate); waits and MMAs from one lane 10.5.  Scores in registers instead of read twice: the same, but 64 single tokens 700 us
// instead of 540 (what the warps that copy had in registers went to memory).
//
// V rows that some row of the item must not see (behind its position, or behind the sequence) would reach it as 0 * V, which is not 0 for
// infinities and NaN.  In the one to three tiles of an item where that can be, two warps take them out of the shared-memory tile: rows
// behind the last visible token whole, other non-finite values one by one; the epilogue adds the latter to the rows that see them.
//
// How items are shared out is decided on the device from the lengths, by every CTA for itself: whole items in rounds of one per CTA
// where there are many, or equal shares of all tiles with a few items split along t, whose parts a second kernel joins.
#include <cuda.h>

#include <algorithm>
#include <type_traits>
#include <vector>

#include "eta_common.cuh"

namespace eta {

constexpr int PF_TILE = 128;               // tokens of a K or V tile
constexpr int PF_HALF = 128;               // query rows of a half item
constexpr int PF_ROWS = 2 * PF_HALF;
constexpr int PF_SOFTMAX_WARPS = 16, PF_WARPS = PF_SOFTMAX_WARPS + 4, PF_THREADS = 32 * PF_WARPS;
constexpr int PF_COPY = PF_SOFTMAX_WARPS, PF_MMA = PF_COPY + 1, PF_CLEAN = PF_MMA + 1;       // warps
constexpr int PF_MAX_CTAS = 160;           // sizes the scratch of split items
constexpr int PF_MAX_BATCH = 1024;         // sequences whose prefix sums a CTA keeps in shared memory
// Cost of a tile of K and V for an item with rows for both halves, for one with rows for one (which streams them); what joining split items
// costs; what an item costs beside its tiles (queries, output, a pipeline that runs dry); in quarter tiles.  A gated tile takes twice as long, so
// an item's own cost is worth half as many of them.  As measured: 64 requests, most of them single tokens, with 4, 3, 2 for the second 1427,
// 1228, 1322 us; with 4, 8, 16, 24, 32 for the last an 8K prompt 644, 605, 558, 579, 586 us, 11 gated prompts 1036, 1034, 1101, 1172, 1205 us.
constexpr int PF_TILE_COST = 4, PF_TWIN_COST = 3, PF_SPLIT_COST = 16;
constexpr int PF_WHOLE_TOKENS = PF_TILE * (PF_SPLIT_COST / PF_TILE_COST);    // no item that sees at most so many tokens is ever split: see PfWalk
template <bool GATED> constexpr int PF_ITEM_COST = GATED ? 8 : 16;
constexpr int64_t PF_L2_BYTES = 64ll << 20;     // K and V of the heads that are worked on side by side
// registers: 640 threads start with 96; 512 of them take 104, the others 64 (together what the block was launched with)
constexpr int PF_REGS = 96, PF_REGS_SOFTMAX = 104, PF_REGS_OTHER = 64;
static_assert(32 * (PF_SOFTMAX_WARPS * PF_REGS_SOFTMAX + 4 * PF_REGS_OTHER) <= PF_REGS * PF_THREADS, "more registers than the block has");
constexpr int PF_CHUNKS = 2;              // weights are handed to the tensor core in so many chunks: of both threads' tokens of a row a part each
constexpr float PF_SLACK = 8.f;            // log2 of how far a weight may exceed 1

struct PrefillArgs {
    const int32_t *row_start, *seq_lens, *granted, *block_table;
    const float *tau, *head_const;
    const __nv_bfloat16* V;                // for values that were taken out of a tile
    int64_t v_sb, v_sh, v_st;
    __nv_bfloat16* out;
    float* part_o;                         // [2 PF_MAX_CTAS][PF_ROWS][D]
    float2* part_ml;                       // [2 PF_MAX_CTAS][PF_ROWS]
    int4* desc;                            // [PF_MAX_CTAS] the split item that starts in a CTA's share: parts, first row, tokens, KV head
    uint32_t* status;
    float a, beta, scale, unit;            // unit: log2 e of what maxima are kept in
    int batch, Hq, Hkv, g_shift, b_shift, t_cap, n_rows, table_stride, n_pages, ungate;
};

// ------------------------------------------------------------------------------------------------ work items

#define PF_BOTH __host__ __device__ __forceinline__

// Tiles of K that query tile t of a sequence needs, and what all before it need, for the n newest of len tokens; m tokens per query tile.
// Where n > len the first rows stand before the sequence's first token and see nothing: query tiles of such rows alone have no tiles.
template <int ITEM_COST>
struct PfTiles {
    int nq, m, n, p0, blind;               // p0: position of the first token; blind: query tiles that see nothing, as far as they are whole
    PF_BOTH PfTiles(int len, int n_, int m_) {
        n = n_; m = m_;
        nq = (n + m - 1) / m;
        p0 = len - n;
        blind = p0 < 0 ? -p0 / m : 0;
    }
    PF_BOTH int tiles(int t) const {
        const int64_t end = p0 + min((int64_t)(t + 1) * m, (int64_t)n);
        return end > 0 ? (int)((end + PF_TILE - 1) / PF_TILE) : 0;
    }
    // what a tile of query tile t counts
    PF_BOTH int weight(int t) const { return t == nq - 1 && 2 * (n - t * m) <= m ? PF_TWIN_COST : PF_TILE_COST; }
    // sum of the tiles of the first t query tiles, t < nq (the last one may be shorter)
    PF_BOTH int64_t before(int t) const {
        t -= blind;
        if (t <= 0) return 0;
        const int64_t b0 = (int64_t)p0 + (int64_t)blind * m + m + PF_TILE - 1;         // at least PF_TILE
        if (m >= PF_TILE) return t * (b0 / PF_TILE) + (int64_t)(m / PF_TILE) * t * (t - 1) / 2;
        const int p = PF_TILE / m, U = t / p, R = t % p;
        int64_t sum = (int64_t)p * U * (U - 1) / 2 + (int64_t)R * U;
        for (int v = 0; v < p; ++v) sum += (int64_t)(U + (v < R)) * ((b0 + v * m) / PF_TILE);
        return sum;
    }
    // cost of the first t query tiles, t <= nq
    PF_BOTH int64_t cost_before(int t) const {
        if (t < nq || !t) return PF_TILE_COST * before(t) + (int64_t)t * ITEM_COST;
        return PF_TILE_COST * before(t - 1) + (int64_t)weight(t - 1) * tiles(t - 1) + (int64_t)t * ITEM_COST;
    }
};

struct PfTables {                          // in shared memory
    int64_t cost[PF_MAX_BATCH + 1];        // cost of all items of the sequences before
    int32_t items[PF_MAX_BATCH + 1];
    int32_t row0[PF_MAX_BATCH], n[PF_MAX_BATCH], len[PF_MAX_BATCH];
    int32_t longest;                       // cost of the longest item's tiles
};

struct PfItem {
    int seq, hk, row0, n_tok;              // first row in the packed rows, tokens that count
    int p0;                                // position of the first token
    int kv_end;                            // tokens [0, kv_end) are seen by some row
    int k0, k1, n0, n1;                    // tiles [k0, k1); how many of them each half takes
    bool twin;                             // rows for one half only: both have them and take turns on the tiles
    int clean0;                            // first tile in which not every row sees every token
    int slot;                              // of a part of a split item; -1: whole
    int pieces;                            // the parts of the item that starts here and goes on; 0: none
    PF_BOTH int n(int half) const { return half ? n1 : n0; }       // (an array indexed by a number would live in memory)
};

// Walks the items of a CTA.  Every warp of it runs the same walk.
template <int ITEM_COST>
struct PfWalk {
    using Tiles = PfTiles<ITEM_COST>;
    const PfTables& tab;
    int batch, Hkv, m, cta, ctas;
    int64_t head_bytes;                    // bytes of K and V per token and KV head
    bool whole;                            // items in rounds, or shares
    int64_t C, x, x1, start;               // shares: all cost, the CTA's range, where the next item starts
    int P, seq, hk, qt;                    // shares; the next item
    int round, total;

    PF_BOTH PfWalk(const PfTables& t, int batch_, int Hkv_, int g_shift, int D, int cta_, int ctas_) : tab(t) {
        batch = batch_; Hkv = Hkv_; m = PF_ROWS >> g_shift;
        cta = cta_; ctas = ctas_;
        head_bytes = 4 * D;
        C = tab.cost[batch];
        total = tab.items[batch];
        round = 0;
        const int64_t longest = tab.longest + ITEM_COST, mean = C / ctas;
        // whole items: as long as the longest, or as the mean with half an item left over at the end
        const int64_t est_whole = total <= ctas ? longest : max(longest, mean + longest / 2);
        whole = est_whole <= mean + ITEM_COST + PF_SPLIT_COST;
        P = (int)min((int64_t)ctas, max((int64_t)1, C / (ITEM_COST + 4 * PF_TILE_COST)));
        x = x1 = C;
        if (whole || cta >= P) return;
        x = C * cta / P; x1 = C * (cta + 1) / P;
        if (x >= x1) return;
        // the item at x; the longest query tile of a head is the first: tile qt lies at [F - cost_before(qt + 1), F - cost_before(qt))
        seq = last_not_above(tab.cost, x);
        const Tiles ti(tab.len[seq], tab.n[seq], m);
        const int64_t F = ti.cost_before(ti.nq), in_seq = x - tab.cost[seq];
        hk = (int)(in_seq / F);
        const int64_t z = F - (in_seq - hk * F);
        int lo = 0, hi = ti.nq;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (ti.cost_before(mid) < z) lo = mid; else hi = mid;
        }
        qt = lo;
        start = tab.cost[seq] + hk * F + F - ti.cost_before(qt + 1);
    }
    template <typename T>
    PF_BOTH int last_not_above(const T* v, T key) const {
        int lo = 0, hi = batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (v[mid] <= key) lo = mid; else hi = mid;
        }
        return lo;
    }
    PF_BOTH void fill(PfItem& it, int seq, int hk, int qt) const {
        const int n = tab.n[seq], len = tab.len[seq], tok = qt * m;
        it.seq = seq; it.hk = hk;
        it.row0 = tab.row0[seq] + tok;
        it.n_tok = min(m, n - tok);
        it.p0 = len - n + tok;
        it.kv_end = max(0, it.p0 + it.n_tok);
        it.clean0 = it.p0 < 0 ? 0 : (it.p0 + 1) / PF_TILE;
    }
    // the part of an item within [k0, k1)
    PF_BOTH void clip(PfItem& it, int k0, int k1) const {
        it.k0 = k0;
        it.k1 = min(k1, it.kv_end > 0 ? (it.kv_end - 1) / PF_TILE + 1 : 0);
        const int n = max(0, it.k1 - k0);
        it.twin = 2 * it.n_tok <= m && n > 1;
        if (it.twin) {
            it.n0 = (n + 1) / 2; it.n1 = n / 2;
            return;
        }
        const int end = it.p0 + min(it.n_tok, m / 2);          // of the first half's rows
        it.n0 = max(0, min(it.k1, end > 0 ? (end - 1) / PF_TILE + 1 : 0) - k0);
        it.n1 = 2 * it.n_tok > m ? n : 0;
    }
    PF_BOTH bool next(PfItem& it) {
        if (whole) {
            // rounds run back and forth, so that whoever got the longest item of one gets the shortest of the next
            while ((int64_t)round * ctas < total) {
                const int idx = round * ctas + ((round & 1) ? ctas - 1 - cta : cta);
                ++round;
                if (idx >= total) continue;
                const int seq = last_not_above(tab.items, idx);
                const Tiles ti(tab.len[seq], tab.n[seq], m);
                // heads in groups whose K and V the L2 holds, within a group the longest query tiles first
                const int group = (int)max((int64_t)1, min((int64_t)Hkv, PF_L2_BYTES / (head_bytes * max(1, tab.len[seq]))));
                int l = idx - tab.items[seq];
                const int g = l / (ti.nq * group);
                l -= g * ti.nq * group;
                const int hs = min(group, Hkv - g * group);
                fill(it, seq, g * group + l % hs, ti.nq - 1 - l / hs);
                clip(it, 0, 1 << 30);
                it.slot = -1; it.pieces = 0;
                return true;
            }
            return false;
        }
        while (x < x1) {
            const Tiles ti(tab.len[seq], tab.n[seq], m);
            const int tiles = ti.tiles(qt), weight = ti.weight(qt);
            const int64_t end = start + ITEM_COST + (int64_t)weight * tiles;
            const int k0 = (int)(max((int64_t)0, x - start - ITEM_COST) / weight);
            const int k1 = (int)(max((int64_t)0, min(x1, end) - start - ITEM_COST) / weight);
            // an item without tiles is done where it starts; of others the share may have no whole tile
            const bool here = k1 > k0 || (!tiles && x == start);
            if (here) {
                fill(it, seq, hk, qt);
                clip(it, k0, k1);
                it.slot = -1; it.pieces = 0;
                if (k0 > 0) {
                    it.slot = 2 * cta;
                } else if (k1 < tiles) {
                    it.slot = 2 * cta + 1;
                    it.pieces = (int)((end * P + C - 1) / C) - cta;          // up to the share that holds the item's last tile
                }
            }
            x = start = end;
            if (--qt < 0) {
                if (++hk == Hkv) {
                    hk = 0;
                    do ++seq; while (seq < batch && !tab.n[seq]);
                }
                if (seq < batch) qt = (tab.n[seq] + m - 1) / m - 1;
            }
            if (here) return true;
        }
        return false;
    }
};

// ------------------------------------------------------------------------------------------------ tensor core

// Operand in shared memory as the copies leave it: rows of 128 bytes, 128-byte swizzle, eight rows (1024 bytes) to a group.
// Queries, keys: the contraction runs along a row.  Values: it runs along the rows, and the next 64 columns are a half tile further.
__device__ __forceinline__ uint64_t pf_operand(uint32_t addr, uint32_t next64) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(next64 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// fp32 accumulator, bf16 operands, 128 rows
__host__ __device__ constexpr uint32_t pf_idesc(int n, bool b_rows) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_rows ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(PF_HALF >> 4) << 24);
}
__device__ __forceinline__ void pf_mma_ss(uint32_t acc, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
__device__ __forceinline__ void pf_mma_ts(uint32_t acc, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(acc), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// arrives on the barrier when every MMA issued so far has completed
__device__ __forceinline__ void pf_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void pf_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pf_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// 32 columns of this thread's lane; complete after pf_wait_ld
__device__ __forceinline__ void pf_ld32(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
          "=r"(r[30]), "=r"(r[31]) : "r"(addr));
}
__device__ __forceinline__ void pf_ld16(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr));
}
__device__ __forceinline__ void pf_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pf_st32(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void pf_st16(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void pf_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float pf_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float pf_max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float pf_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pf_pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// (a0, a1) * (b, b) + (c, c)
__device__ __forceinline__ void pf_fma2(float& d0, float& d1, float a0, float a1, float b, float c) {
    asm("{\n\t.reg .b64 ra, rb, rc;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %4};\n\tmov.b64 rc, {%5, %5};\n\t"
        "fma.rn.f32x2 rc, ra, rb, rc;\n\tmov.b64 {%0, %1}, rc;\n\t}"
        : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c));
}

__device__ __forceinline__ bool pf_elect() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// Whether q holds for any thread of the N warps that share barrier `id`, which meet here
template <int N>
__device__ __forceinline__ bool pf_any_of(bool q, int id) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, o;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred o, %2, %3, p;\n\tselp.u32 %0, 1, 0, o;\n\t}"
                 : "=r"(r) : "r"((uint32_t)q), "r"(id), "n"(32 * N) : "memory");
    return r != 0;
}

// A bounded wait that others' failures end too
__device__ __forceinline__ bool pf_wait(uint64_t* bar, uint32_t parity, const volatile int* dead) {
    for (uint32_t it = 0; it < WAIT_LIMIT; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 255) == 255 && *dead) return false;
    }
    return false;
}

// ------------------------------------------------------------------------------------------------ kernel

template <int D>
struct PfSmem {
    static constexpr int HALVES = D / 64;
    static constexpr int Q_BYTES = PF_HALF * D * 2;
    static constexpr int STAGE = PF_TILE * D * 2;
    static constexpr int NSTAGE = 128 * 1024 / STAGE;
    static constexpr int RING = 2 * Q_BYTES;
    static constexpr int TABLES = RING + NSTAGE * STAGE;
    static constexpr int BARS = TABLES + (int)((sizeof(PfTables) + 15) / 16 * 16);
    static constexpr int N_BARS = 3 * NSTAGE + 2 * (4 + PF_CHUNKS) + 1 + 4;
    static constexpr int BYTES = 1024 + BARS + 8 * N_BARS;
    static_assert(PF_CHUNKS == 2, "a chunk is 32 of a thread's columns");
    static_assert(BYTES <= 227 * 1024, "too much shared memory");
};

template <int D, bool GATED>
__global__ void __launch_bounds__(PF_THREADS, 1)
prefill_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
               const __grid_constant__ PrefillArgs a) {
    using L = PfSmem<D>;
    constexpr int NSTAGE = L::NSTAGE, HALVES = L::HALVES;
    extern __shared__ unsigned char pf_raw[];
    unsigned char* const smem = pf_raw + ((1024u - (smem_u32(pf_raw) & 1023u)) & 1023u);
    PfTables& tab = *reinterpret_cast<PfTables*>(smem + L::TABLES);
    uint64_t* const full = reinterpret_cast<uint64_t*>(smem + L::BARS);
    uint64_t *const empty = full + NSTAGE, *const cleaned = empty + NSTAGE;
    uint64_t *const q_full = cleaned + NSTAGE, *const q_empty = q_full + 2, *const s_full = q_empty + 2, *const p_full = s_full + 2,
             *const o_full = p_full + 2 * PF_CHUNKS, *const drained = o_full + 2, *const handed = drained + 1;
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    // The item of whose tiles values were taken out, of those with tiles, counted from 1.  The cleaning warps are no more such items ahead of the
    // epilogue than the ring has tiles.
    __shared__ int s_poison[16];
    static_assert(NSTAGE / 2 + 1 < 16, "an item's mark would be overwritten before it is read");
    __shared__ int64_t s_scan[PF_WARPS][2];
    __shared__ float s_x[2][PF_ROWS];          // what the two threads of a row tell each other
    __shared__ float2 s_twin[PF_HALF];         // maximum and sum of a twin item's second half

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = 1 << a.g_shift, HT = PF_HALF >> a.g_shift;       // heads of a group, tokens of a half

    if (tid == 0) {
        // (tiles of K and V take turns, so the odd stages hold V: the cleaning warps let go of those too)
        for (int k = 0; k < NSTAGE; ++k) { mbar_init(&full[k], 1); mbar_init(&empty[k], k & 1 ? 3 : 1); mbar_init(&cleaned[k], 2); }
        mbar_init(drained, 1);
        for (int k = 0; k < 4; ++k) mbar_init(&handed[k], 2);
        for (int k = 0; k < 2; ++k) {
            mbar_init(&q_full[k], 1); mbar_init(&q_empty[k], 1 + PF_SOFTMAX_WARPS / 2); mbar_init(&s_full[k], 1);
            for (int c = 0; c < PF_CHUNKS; ++c) mbar_init(&p_full[k * PF_CHUNKS + c], PF_SOFTMAX_WARPS / 2);
            mbar_init(&o_full[k], 1);
        }
        fence_barrier_init();
        prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
        s_dead = 0;
        tab.longest = 0;
    }
    if (tid < 16) s_poison[tid] = 0;
    if (warp == PF_MMA) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    __syncthreads();

    // ---- sequences: rows, lengths, and prefix sums of items and cost
    {
        const int per = (a.batch + PF_THREADS - 1) / PF_THREADS, first = min(a.batch, tid * per), end = min(a.batch, first + per);
        int64_t cost = 0;
        int items = 0, longest = 0;
        uint32_t flags = 0;
        for (int i = first; i < end; ++i) {
            const int r0 = __ldcg(a.row_start + i), r1 = __ldcg(a.row_start + i + 1);
            int len = __ldcg(a.seq_lens + i), n = r1 > r0 ? r1 - r0 : 0;
            if (a.granted) n = min(n, max(0, __ldcg(a.granted + i)));
            if (r0 < 0 || r0 > a.n_rows) n = 0;
            n = min(n, a.n_rows - min(max(r0, 0), a.n_rows));
            if (len > a.t_cap) { len = a.t_cap; flags |= ETA_DEV_LEN_CLAMPED; }
            len = max(len, 0);
            if (n > len) flags |= ETA_DEV_EMPTY_ROW;
            tab.row0[i] = r0; tab.n[i] = n; tab.len[i] = len;
            tab.items[i] = items; tab.cost[i] = cost;
            const PfTiles<PF_ITEM_COST<GATED>> ti(len, n, PF_ROWS >> a.g_shift);
            items += ti.nq * a.Hkv;
            cost += a.Hkv * ti.cost_before(ti.nq);
            if (n) longest = max(longest, ti.weight(ti.nq - 1) * ti.tiles(ti.nq - 1));
            if (ti.nq > 1) longest = max(longest, PF_TILE_COST * ti.tiles(ti.nq - 2));
        }
        int64_t sc = cost, si = items;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t oc = __shfl_up_sync(0xffffffffu, sc, s), oi = __shfl_up_sync(0xffffffffu, si, s);
            if (lane >= s) { sc += oc; si += oi; }
        }
        if (lane == 31) { s_scan[warp][0] = sc; s_scan[warp][1] = si; }
        longest = __reduce_max_sync(0xffffffffu, longest);
        if (lane == 0 && longest) atomicMax(&tab.longest, longest);
        flags = __reduce_or_sync(0xffffffffu, flags);
        if (lane == 0 && flags && blockIdx.x == 0 && a.status) atomicOr(a.status, flags);
        __syncthreads();
        sc -= cost; si -= items;
        for (int w = 0; w < warp; ++w) { sc += s_scan[w][0]; si += s_scan[w][1]; }
        for (int i = first; i < end; ++i) { tab.cost[i] += sc; tab.items[i] += (int)si; }
        if (end == a.batch && first < end) { tab.cost[a.batch] = sc + cost; tab.items[a.batch] = (int)si + items; }
    }
    pf_fence_before();
    __syncthreads();
    pf_fence_after();
    const uint32_t tmem = s_tmem;
    PfWalk<PF_ITEM_COST<GATED>> walk(tab, a.batch, a.Hkv, a.g_shift, D, blockIdx.x, gridDim.x);
    PfItem it;
    bool ok = true;
    // Said by every warp whose wait ran out: those that the others wait for may have done their work by then.
    auto gave_up = [&] {
        if (ok || lane) return;
        s_dead = 1;
        if (a.status) atomicOr(a.status, ETA_DEV_TIMEOUT);
    };

    if (warp >= PF_SOFTMAX_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PF_REGS_OTHER));
        if (warp == PF_COPY) {
            // -------------------------------------------------------------- copies
            uint32_t fill = 0, q_par = 0, q_some = 0;          // a bit per half: the parity of its next load, whether there was one
            auto wait = [&](uint64_t* bar, uint32_t parity) {  // (the same answer in all lanes)
                return ok = __all_sync(0xffffffffu, pf_wait(bar, parity, &s_dead));
            };
            int4 split = make_int4(0, 0, 0, 0);
            while (ok && walk.next(it)) {
                if (it.pieces > 1) split = make_int4(it.pieces, it.row0, it.n_tok, it.hk);
                const int n = max(0, it.k1 - it.k0);
                auto load_q = [&](int h) {
                    if (!ok || !it.n(h)) return;
                    if (((q_some >> h) & 1) && !wait(&q_empty[h], ((q_par >> h) & 1) ^ 1)) return;
                    q_some |= 1u << h;
                    q_par ^= 1u << h;
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&q_full[h], L::Q_BYTES);
#pragma unroll
                        for (int c = 0; c < HALVES; ++c)
                            asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                                         ::"r"(smem_u32(smem + h * L::Q_BYTES + c * (PF_HALF * 128))), "l"(&tmQ), "r"(smem_u32(&q_full[h])),
                                           "r"(64 * c), "r"(it.hk * G), "r"(it.row0 + (it.twin ? 0 : h * HT)) : "memory");
                    }
                    __syncwarp();
                };
                // a tile: a copy per 64 columns, and in a paged cache per page
                const int per_tile = a.block_table ? PF_TILE >> a.b_shift : 1;
                auto load_tile = [&](const CUtensorMap* tm, int j, int page) {
                    if (!ok) return;
                    const int stage = fill % NSTAGE;
                    if (!wait(&empty[stage], ((fill / NSTAGE) & 1) ^ 1)) return;
                    ++fill;
                    int copies = HALVES, bytes = L::STAGE;
                    if (a.block_table) {
                        const int pages = (min(PF_TILE, it.kv_end - j * PF_TILE) + (1 << a.b_shift) - 1) >> a.b_shift;
                        copies = HALVES * pages;
                        bytes = (pages << a.b_shift) * D * 2;
                    }
                    if (lane == 0) mbar_arrive_expect_tx(&full[stage], bytes);
                    __syncwarp();
                    const int sub = lane / HALVES, c = lane % HALVES;
                    if (lane < copies)
                        tma_load_4d(smem + L::RING + stage * L::STAGE + c * (PF_TILE * 128) + ((sub << a.b_shift) * 128 & (PF_TILE * 128 - 1)), tm, 64 * c,
                                    a.block_table ? 0 : j * PF_TILE, it.hk, a.block_table ? page : it.seq, &full[stage]);
                    __syncwarp();
                };
                auto page_of = [&](int j) {            // the page of this lane's copy
                    const int sub = lane / HALVES, blk = j * per_tile + sub;
                    return a.block_table && sub < per_tile && (blk << a.b_shift) < it.kv_end
                               ? __ldcg(a.block_table + (int64_t)it.seq * a.table_stride + blk) : 0;
                };
                int page = n ? page_of(it.k0) : 0;
                load_q(0);
                for (int j = 0; j < n && ok; ++j) {
                    const int next = j + 1 < n ? page_of(it.k0 + j + 1) : 0;
                    load_tile(&tmK, it.k0 + j, page);
                    if (j == 0) load_q(1);
                    load_tile(&tmV, it.k0 + j, page);
                    page = next;
                }
            }
            if (lane == 0) a.desc[blockIdx.x] = split;
            pdl_trigger();
            gave_up();
            // The copies that are on their way land before the shared memory is given back: whoever they are for may have given up, or may yet.
            for (uint32_t f = fill > NSTAGE ? fill - NSTAGE : 0; f < fill; ++f) mbar_wait(&full[f % NSTAGE], (f / NSTAGE) & 1);
            for (int h = 0; h < 2; ++h)
                if ((q_some >> h) & 1) mbar_wait(&q_full[h], ((q_par >> h) & 1) ^ 1);
        } else if (warp == PF_MMA) {
            // -------------------------------------------------------------- MMAs; the whole warp walks along, one lane issues
            // Every instruction between a wait and the MMAs behind it is time that the tensor core stands still: the warp takes some seven
            // cycles for one.
            uint32_t fill = 0, n_clean = 0, q_par = 0, p_par = 0;          // (parities: a bit per half)
            const uint64_t q_op0 = pf_operand(smem_u32(smem), 16), ring_k = pf_operand(smem_u32(smem + L::RING), 16),
                           ring_v = pf_operand(smem_u32(smem + L::RING), PF_TILE * 128);
            auto wait = [&](uint64_t* bar, uint32_t parity) {              // (the same answer in all lanes)
                for (uint32_t it_ = 0; it_ < WAIT_LIMIT; ++it_) {
                    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
                    if ((it_ & 255) == 255 && __any_sync(0xffffffffu, *(volatile int*)&s_dead)) break;
                }
                ok = false;
                return false;
            };
            auto there = [&](uint32_t f) { return wait(&full[f % NSTAGE], (f / NSTAGE) & 1); };
            // One turn of half h: O += P V with the values of fill fv, then S = Q K^T with the keys of fill fk, over the weights; the latter goes
            // out right behind the former.  What both read has been waited for.
            enum { VALUES = 1, KEYS = 2, FIRST = 4, LAST_VALUES = 8, LAST_KEYS = 16, FREE_VALUES = 32, FREE_KEYS = 64 };
            auto turn = [&](int h, uint32_t fv, uint32_t fk, uint32_t what) {
                const uint64_t q_op = q_op0 + (uint32_t)(h * (L::Q_BYTES >> 4)), k_op = ring_k + (fk % NSTAGE) * (L::STAGE >> 4);
                const uint64_t v_op = ring_v + (fv % NSTAGE) * (L::STAGE >> 4);
                const uint32_t t_s = h * PF_TILE, t_o = 2 * PF_TILE + h * D, parity = (p_par >> h) & 1;
                constexpr int PER = PF_TILE / 32 / PF_CHUNKS;
                auto values = [&](int c) {
#pragma unroll
                    for (int u = 0; u < 2 * PER; ++u) {        // 16 tokens: two groups of eight rows; a chunk's share of the first 64 tokens, then of the others
                        const int k = c * PER + u % PER + (u / PER) * (PF_TILE / 32);
                        pf_mma_ts(t_o, t_s + 8 * k + (k >= PF_TILE / 32 ? PF_TILE / 4 : 0), v_op + k * (16 * 128 >> 4), pf_idesc(D, true), !(what & FIRST) || c > 0 || u > 0);
                    }
                };
                if (what & VALUES) {
#pragma unroll
                    for (int c = 0; c + 1 < PF_CHUNKS; ++c) {
                        if (!wait(&p_full[h * PF_CHUNKS + c], parity)) return;
                        pf_fence_after();
                        if (pf_elect()) values(c);
                    }
                    if (!wait(&p_full[h * PF_CHUNKS + PF_CHUNKS - 1], parity)) return;
                    pf_fence_after();
                    p_par ^= 1u << h;
                }
                if (pf_elect()) {
                    if (what & VALUES) values(PF_CHUNKS - 1);
                    if (what & KEYS) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)       // 16 columns: 32 bytes along the swizzled row of a 64-column half
                            pf_mma_ss(t_s, q_op + (k / 4) * (PF_HALF * 128 >> 4) + (k % 4) * 2, k_op + (k / 4) * (PF_TILE * 128 >> 4) + (k % 4) * 2,
                                      pf_idesc(PF_TILE, false), k > 0);
                        pf_commit(&s_full[h]);
                    }
                    bool last = what & LAST_VALUES;
#ifdef ETA_TEST_SKIP_LAST_COMMIT
                    last = last && (blockIdx.x != 1 || it.twin || it.n1);              // (an item of the first half only)
#endif
                    if (last) pf_commit(&o_full[h]);
                    if (what & LAST_KEYS) pf_commit(&q_empty[h]);
                    if (what & FREE_VALUES) pf_commit(&empty[fv % NSTAGE]);
                    if (what & FREE_KEYS) pf_commit(&empty[fk % NSTAGE]);
                }
                __syncwarp();
            };
            while (ok && walk.next(it)) {
                const int n = max(0, it.k1 - it.k0), step = it.twin ? 2 : 1;
                // tile j: keys in fill base + 2 j, values in the one behind it
                const uint32_t base = fill;
                fill += 2 * n;
                const int last_half = it.twin || it.n1 == 0 ? 0 : 1;       // whose turn frees a tile's stages (not twin)
#pragma unroll 1
                for (int h = 0; h < 2 && ok; ++h) {
                    const uint32_t f = base + (it.twin ? 2 * h : 0);
                    if (!it.n(h) || !wait(&q_full[h], (q_par >> h) & 1)) continue;
                    q_par ^= 1u << h;
                    if (there(f)) turn(h, 0, f, KEYS | (it.n(h) == 1 ? LAST_KEYS : 0) | (it.twin || h == last_half ? FREE_KEYS : 0));
                }
                for (int j = 0; j < n && ok; ++j) {
                    const uint32_t f = base + 2 * j + 1, next = base + 2 * (j + step);
                    const bool more = j + step < n;
                    if (!there(f)) break;
                    if (it.k0 + j >= it.clean0) {
                        if (!wait(&cleaned[n_clean % NSTAGE], (n_clean / NSTAGE) & 1)) break;
                        ++n_clean;
                    }
                    // (where memory is slow the next keys are not there yet: products first then)
                    const bool ready = more && __all_sync(0xffffffffu, mbar_test(&full[next % NSTAGE], (next / NSTAGE) & 1));
                    // half after half, so that one half's weights are worked out while the other's products run
#pragma unroll 1
                    for (int h = it.twin ? j & 1 : 0; h < 2 && ok; h += step) {
                        const int i = it.twin ? j >> 1 : j, left = it.n(h) - i;        // steps of the half that are left, this one among them
                        if (left <= 0) continue;
                        const bool frees = it.twin || h == last_half;
                        const uint32_t v = VALUES | (i == 0 ? FIRST : 0) | (left == 1 ? LAST_VALUES : 0) | (frees ? FREE_VALUES : 0);
                        const uint32_t k = left > 1 ? KEYS | (left == 2 ? LAST_KEYS : 0) | (frees ? FREE_KEYS : 0) : 0;
                        turn(h, f, next, ready ? v | k : v);
                        if (k && !ready && ok && there(next)) turn(h, 0, next, k);
                    }
                }
            }
            // what was issued has to end before tensor and shared memory are given back
            if (pf_elect()) pf_commit(drained);
            __syncwarp();
            ok = __all_sync(0xffffffffu, mbar_wait(drained, 0)) && ok;
            gave_up();
        } else {
            // -------------------------------------------------------------- values that not every row may see
            uint32_t fill = 0, n_clean = 0;
            int item = 0;
            const int w = warp - PF_CLEAN;             // which half of the tile's rows
            while (ok && walk.next(it)) {
                const int n = max(0, it.k1 - it.k0);
                item += n > 0;
                for (int j = 0; j < n; ++j) {
                    ++fill;                            // K's
                    const int stage = fill % NSTAGE;
                    ok = __all_sync(0xffffffffu, pf_wait(&full[stage], (fill / NSTAGE) & 1, &s_dead));
                    if (!ok) break;
                    ++fill;
                    if (it.k0 + j >= it.clean0) {
                        bool found = false;
                        unsigned char* const tile = smem + L::RING + stage * L::STAGE + w * (PF_TILE / 2 * 128) + lane * 16;
                        const int t0 = (it.k0 + j) * PF_TILE + w * (PF_TILE / 2) + (lane >> 3);
#pragma unroll 4
                        for (int r = 0; r < PF_TILE / 2; r += 4)
#pragma unroll
                            for (int c = 0; c < HALVES; ++c) {
                                uint4* const at = reinterpret_cast<uint4*>(tile + c * (PF_TILE * 128) + r * 128);
                                if (t0 + r >= it.kv_end) {
                                    *at = make_uint4(0, 0, 0, 0);
                                    continue;
                                }
                                uint4 v = *at;
                                // an exponent of all ones carries into the sign's place
                                auto non_finite = [](uint32_t x) { return (x & 0x7f807f80u) + 0x00800080u; };
                                if ((non_finite(v.x) | non_finite(v.y) | non_finite(v.z) | non_finite(v.w)) & 0x80008000u) {
                                    uint32_t* const x = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                                    for (int u = 0; u < 4; ++u) {
                                        const uint32_t bad = non_finite(x[u]);
                                        x[u] &= ~(((bad >> 31) * 0xffff0000u) | (((bad >> 15) & 1u) * 0xffffu));
                                    }
                                    *at = v;
                                    found = true;
                                }
                            }
                        if (found) s_poison[item & 15] = item;
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&cleaned[n_clean % NSTAGE]);
                        ++n_clean;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&empty[stage]);
                }
            }
            gave_up();
        }
    } else {
        // ------------------------------------------------------------------ softmax and epilogue: two threads to a row, 64 tokens of a
        // tile and half of head_dim each
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PF_REGS_SOFTMAX));
        constexpr float LOG2E = 1.4426950408889634f;
        constexpr int W = PF_TILE / 2, DW = D / 2;
        const int half = (warp >> 2) & 1, part = warp >> 3, wrow = (warp & 3) * 32, row = wrow + lane;
        const uint32_t lanes = (uint32_t)wrow << 16;
        const uint32_t t_s = tmem + lanes + half * PF_TILE + part * W;
        const uint32_t t_o = tmem + lanes + 2 * PF_TILE + half * D + part * DW;
        const int pair = 1 + (warp & 7);               // the barrier of the two warps that share 32 rows
        float* const tell = &s_x[part][half * PF_HALF + row];
        const float* const told = &s_x[part ^ 1][half * PF_HALF + row];
        const float sl2 = a.scale * LOG2E, kb = a.scale * a.beta * LOG2E, unit = GATED ? 1.f : sl2;
        uint32_t s_n = 0, o_n = 0, h_n = 0;
        int item = 0;
        while (ok && walk.next(it)) {
            item += it.k1 > it.k0;
            const int tok0 = it.twin ? 0 : half * HT, rows = min(max(it.n_tok - tok0, 0), HT) << a.g_shift;
            if (!rows) continue;
            const int n = it.n(half);
            const bool live = wrow < rows;                  // a warp without rows only keeps step
            const int r = min(row, rows - 1), tok = tok0 + (r >> a.g_shift), h = it.hk * G + (r & (G - 1));
            const int p = it.p0 + tok;                      // the row sees tokens 0 .. p
            float tb = 0.f;                                 // the gate is 1 / (1 + 2^(tb - kb q.k))
            float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
            if (GATED && live) {
                const float tau = a.tau ? __ldcg(a.tau + (int64_t)(it.row0 + tok) * a.Hq + h) : __ldcg(a.head_const + h);
                const float te = tau - a.a;
                if (a.beta != 0.f) tb = te * a.beta * LOG2E;
                if (te != te) l0 = te;                      // a threshold that is NaN: so is the row
            }
            float m = -INFINITY;                            // running maximum, of q.k (gated: of S~ log2 e)
            for (int j = 0; j < n; ++j) {
                ok = __all_sync(0xffffffffu, pf_wait(&s_full[half], s_n++ & 1, &s_dead));
                if (j == 0 && !it.twin && lane == 0) mbar_arrive(&q_empty[half]);
                if (live) {
                    pf_fence_after();
                    // The scores are read twice, 32 columns at a time: for the maximum (gated ones, and those at an edge, go back to where they
                    // came from), then for the weights, which take the place of the first half of them.
                    const int tile = it.k0 + (it.twin ? 2 * j + half : j);
                    const int nvis = p - tile * PF_TILE - part * W + 1;                  // columns that the row sees
                    const bool edge = __any_sync(0xffffffffu, nvis <= W);
                    float mx = -INFINITY;
#pragma unroll 1
                    for (int g = 0; g < 2; ++g) {
                        float s[32];
                        pf_ld32(t_s + 32 * g, s);
                        const int here = nvis - 32 * g;
                        pf_wait_ld();
                        if constexpr (GATED) {
                            // what the row does not see is out before anything is taken of several columns together
                            if (edge) {
#pragma unroll
                                for (int k = 0; k < 32; ++k) s[k] = k < here ? s[k] : 0.f;
                            }
                            const int own = a.ungate ? here - 1 : -1;             // the column that stays raw
                            float am[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int k = 0; k < 32; k += 8)
#pragma unroll
                                for (int u = 0; u < 4; ++u) am[u] = pf_max3(am[u], fabsf(s[k + u]), fabsf(s[k + u + 4]));
                            auto exact = [&](float sk) { return sk * sl2 * pf_rcp(1.f + pf_ex2(fmaf(sk, -kb, tb))); };
                            auto eight = [&](int k0) {                         // stage by stage, so that chains run side by side
                                float x[8], e[8], r[4];
#pragma unroll
                                for (int k = 0; k < 8; k += 2) pf_fma2(e[k], e[k + 1], s[k0 + k], s[k0 + k + 1], -kb, tb);
                                // The reciprocals of four from the one of their product.  So that it stays finite a gate is no smaller than
                                // 2^-31: a score below 2^11 then counts as 0 all the same (2^-20 of a weight).
#pragma unroll
                                for (int k = 0; k < 8; ++k) e[k] = pf_ex2(fminf(e[k], 31.f));
#pragma unroll
                                for (int k = 0; k < 8; k += 2) { add2(e[k], e[k + 1], 1.f, 1.f); mul2(x[k], x[k + 1], s[k0 + k], s[k0 + k + 1], sl2, sl2); }
#pragma unroll
                                for (int k = 0; k < 8; k += 4) {
                                    const float p0 = e[k] * e[k + 1], p1 = e[k + 2] * e[k + 3], both = pf_rcp(p0 * p1);
                                    r[k / 2] = both * p1;
                                    r[k / 2 + 1] = both * p0;
                                }
#pragma unroll
                                for (int k = 0; k < 8; k += 2) mul2(e[k + 1], e[k], x[k], x[k + 1], e[k + 1], e[k]);
#pragma unroll
                                for (int k = 0; k < 8; k += 2) mul2(s[k0 + k], s[k0 + k + 1], e[k + 1], e[k], r[k / 2], r[k / 2]);
                                if (edge) {
#pragma unroll
                                    for (int k = 0; k < 8; ++k) s[k0 + k] = k0 + k == own ? x[k] : s[k0 + k];
                                }
                            };
                            // Which of the two a thread's scores take is a matter of its own row: a row's bits do not hang on its neighbours.
                            const bool large = !(pf_max3(fmaxf(am[0], am[1]), am[2], am[3]) * sl2 < 0x1p11f);
                            if (__any_sync(0xffffffffu, large)) {
#pragma unroll
                                for (int k0 = 0; k0 < 32; k0 += 8) {
                                    float y[8];
#pragma unroll
                                    for (int k = 0; k < 8; ++k) y[k] = k0 + k == own ? s[k0 + k] * sl2 : exact(s[k0 + k]);
                                    eight(k0);
#pragma unroll
                                    for (int k = 0; k < 8; ++k) s[k0 + k] = large ? y[k] : s[k0 + k];
                                }
                            } else {
#pragma unroll
                                for (int k0 = 0; k0 < 32; k0 += 8) eight(k0);
                            }
                        }
                        if (edge) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) s[k] = k < here ? s[k] : -INFINITY;
                        }
                        if (GATED || edge) pf_st32(t_s + 32 * g, reinterpret_cast<const uint32_t*>(s));
                        float x[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[k] = pf_max3(s[k], s[k + 4], s[k + 8]);
#pragma unroll
                        for (int k = 12; k + 8 <= 32; k += 8)
#pragma unroll
                            for (int u = 0; u < 4; ++u) x[u] = pf_max3(x[u], s[k + u], s[k + u + 4]);
                        mx = pf_max3(mx, pf_max3(pf_max3(x[0], x[1], x[2]), x[3], s[28]), pf_max3(s[29], s[30], s[31]));
                    }
                    if (GATED || edge) pf_wait_st();
                    // Both threads meet here.  A warp whose wait ran out comes here too, so that no meeting is left waiting for it.
                    if (pf_any_of<2>(!ok || (mx - m) * unit > PF_SLACK, pair)) {
                        *tell = mx;
                        if (pf_any_of<2>(!ok, pair)) { ok = false; break; }
                        mx = fmaxf(mx, *told);
                        const float m_new = (mx - m) * unit > PF_SLACK ? mx : m;      // (by the row's own scores, whoever of the others asked for it)
                        const float alpha = m == m_new ? 1.f : pf_ex2((m - m_new) * unit);
                        m = m_new;
                        l0 *= alpha; l1 *= alpha; l2 *= alpha; l3 *= alpha;
                        if (j) {                       // these scores are complete, so is the product before them
#pragma unroll 1
                            for (int k = 0; k < DW; k += 16) {
                                float o[16];
                                pf_ld16(t_o + k, o);
                                pf_wait_ld();
#pragma unroll
                                for (int u = 0; u < 16; ++u) o[u] *= alpha;
                                pf_st16(t_o + k, reinterpret_cast<const uint32_t*>(o));
                            }
                        }
                    }
                    // The difference first: scores of any size lose nothing next to the largest.
                    const float minus = m == -INFINITY ? 0.f : -m;
#pragma unroll 1
                    for (int g = 0; g < PF_CHUNKS; ++g) {
                        float s[32];
                        uint32_t w[16];
                        pf_ld32(t_s + 32 * g, s);
                        pf_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; k += 2) {
                            add2(s[k], s[k + 1], minus, minus);
                            if (!GATED) mul2(s[k], s[k + 1], s[k], s[k + 1], sl2, sl2);
                        }
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
#pragma unroll
                            for (int u = 0; u < 8; ++u) s[k + u] = pf_ex2(s[k + u]);
#pragma unroll
                            for (int u = 0; u < 8; u += 4) {
                                add2(l0, l1, s[k + u], s[k + u + 1]);
                                add2(l2, l3, s[k + u + 2], s[k + u + 3]);
                                w[(k + u) / 2] = pf_pack(s[k + u], s[k + u + 1]);
                                w[(k + u) / 2 + 1] = pf_pack(s[k + u + 2], s[k + u + 3]);
                            }
                        }
                        pf_st16(t_s + 16 * g, w);
                        pf_wait_st();
                        pf_fence_before();
                        __syncwarp();
                        bool hands_over = lane == 0;
#ifdef ETA_TEST_SKIP_WEIGHTS_ARRIVE
                        hands_over = hands_over && (blockIdx.x || warp != 4);          // (a warp of the second half)
#endif
                        if (hands_over) mbar_arrive(&p_full[half * PF_CHUNKS + g]);
                    }
                } else {
                    if (!ok) break;
                    if (lane == 0)
                        for (int k = 0; k < PF_CHUNKS; ++k) mbar_arrive(&p_full[half * PF_CHUNKS + k]);
                }
            }
            if (!ok) break;
            if (n) ok = __all_sync(0xffffffffu, pf_wait(&o_full[half], o_n++ & 1, &s_dead));
            pf_fence_after();
            const bool mine = row < rows, split = it.slot >= 0;
            const int64_t at_part = ((int64_t)it.slot * PF_ROWS + (it.twin ? 0 : half * PF_HALF) + row);
            // In a twin item both halves have the row: the second hands over what it has, through the queries' place (a column's rows side by side).
            float* const hand = reinterpret_cast<float*>(smem) + part * DW * PF_HALF + row;
            float l = (l0 + l1) + (l2 + l3), keep = 1.f, take = 0.f;               // what either half's sums count
            // Without tiles there is nothing to tell (l is the same in both threads), and it would be told over what a slow partner has yet to read of
            // the item before: only items with tiles meet again, at their first maximum, before the next of them is told anything.
            if (live && n) {
                // The two warps of a row agree on whether a wait ran out: what both have waited for comes before they meet.  Halves do not meet: one may
                // have left over an earlier item.
                if (it.twin && !half && ok) ok = __all_sync(0xffffffffu, pf_wait(&handed[warp & 3], h_n++ & 1, &s_dead));
                *tell = l;
                if (pf_any_of<2>(!ok, pair)) ok = false;
                l = part ? *told + l : l + *told;
                if (it.twin && ok) {
                    if (half) {
#pragma unroll 1
                        for (int k = 0; k < DW; k += 16) {
                            float o[16];
                            pf_ld16(t_o + k, o);
                            pf_wait_ld();
#pragma unroll
                            for (int u = 0; u < 16; ++u) hand[(k + u) * PF_HALF] = o[u];
                        }
                        if (!part) s_twin[row] = make_float2(m, l);
                        pf_fence_before();
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&handed[warp & 3]);
                    } else {
                        const float2 ml = s_twin[row];
                        const float M = fmaxf(m, ml.x);
                        if (M != -INFINITY) { keep = pf_ex2((m - M) * unit); take = pf_ex2((ml.x - M) * unit); }
                        l = l * keep + ml.y * take;
                        m = M;
                    }
                }
            }
            if (!ok) break;
            const bool poison = n && s_poison[item & 15] == item;
            if (split && live && mine && !part && !(it.twin && half)) a.part_ml[at_part] = make_float2(m, l);
            const float inv = split ? 1.f : (l == 0.f ? 0.f : 1.f / l);
            keep *= inv; take *= inv;
            const int64_t to = ((int64_t)(it.row0 + tok) * a.Hq + h) * D + part * DW;
#pragma unroll 1
            for (int k = 0; k < (live && !(it.twin && half) ? DW : 0); k += 32) {
                float o[32];
                if (n) {
                    pf_ld32(t_o + k, o);
                    pf_wait_ld();
#pragma unroll
                    for (int u = 0; u < 32; ++u) o[u] *= keep;
                    if (it.twin) {
#pragma unroll
                        for (int u = 0; u < 32; ++u) o[u] = fmaf(hand[(k + u) * PF_HALF], take, o[u]);
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < 32; ++u) o[u] = 0.f;
                }
                if (poison) {
                    const int end = (int)min((int64_t)p + 1, (int64_t)it.k1 * PF_TILE);
                    for (int t = max(it.clean0, it.k0) * PF_TILE; t < end; ++t) {
                        int64_t base = (int64_t)it.seq * a.v_sb + (int64_t)t * a.v_st;
                        if (a.block_table) {
                            const int page = __ldcg(a.block_table + (int64_t)it.seq * a.table_stride + (t >> a.b_shift));
                            if (page < 0 || page >= a.n_pages) continue;       // the copies read zeros there
                            base = (int64_t)page * a.v_sb + (int64_t)(t & ((1 << a.b_shift) - 1)) * a.v_st;
                        }
                        const uint4* const from = reinterpret_cast<const uint4*>(a.V + base + it.hk * a.v_sh + part * DW + k);
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const uint4 v = __ldcg(from + u);
                            const uint32_t x4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const float lo = bf16_lo(x4[q]), hi = bf16_hi(x4[q]);
                                if (!isfinite(lo)) o[8 * u + 2 * q] += lo;
                                if (!isfinite(hi)) o[8 * u + 2 * q + 1] += hi;
                            }
                        }
                    }
                }
                if (!mine) continue;
                if (split) {
                    float4* const at = reinterpret_cast<float4*>(a.part_o + at_part * D + part * DW + k);
#pragma unroll
                    for (int u = 0; u < 8; ++u) at[u] = make_float4(o[4 * u], o[4 * u + 1], o[4 * u + 2], o[4 * u + 3]);
                } else {
                    uint4* const at = reinterpret_cast<uint4*>(a.out + to + k);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        at[u] = make_uint4(pf_pack(o[8 * u], o[8 * u + 1]), pf_pack(o[8 * u + 2], o[8 * u + 3]), pf_pack(o[8 * u + 4], o[8 * u + 5]),
                                           pf_pack(o[8 * u + 6], o[8 * u + 7]));
                }
            }
            pf_fence_before();
            if (it.twin && !half) {                        // all is read: the next item's queries may come
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) { mbar_arrive(&q_empty[0]); mbar_arrive(&q_empty[1]); }
            }
        }
        gave_up();
        pdl_trigger();
    }
    pf_fence_before();
    __syncthreads();
    if (warp == PF_MMA) {
        pf_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// Joins the parts of split items, in the order of their tiles.  A CTA per (share in which a split item starts, 32 of its rows), a warp per row.
constexpr int PF_JOIN_ROWS = 32, PF_JOIN_WARPS = 8;
template <int D>
__global__ void __launch_bounds__(32 * PF_JOIN_WARPS) prefill_join_kernel(const __grid_constant__ PrefillArgs a) {
    const int cta = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    const int4 d = __ldcg(a.desc + cta);
    const int pieces = d.x, rows = d.z << a.g_shift, G = 1 << a.g_shift;
    if (pieces < 2) return;
    constexpr int PER = D / 32;
    for (int r = blockIdx.y * PF_JOIN_ROWS + warp; r < min(rows, (int)(blockIdx.y + 1) * PF_JOIN_ROWS); r += PF_JOIN_WARPS) {
        // the first part is the second slot of its share, the others the first of theirs
        auto slot = [&](int k) { return (int64_t)(2 * (cta + k) + (k == 0)) * PF_ROWS + r; };
        float M = -INFINITY;
        for (int k = lane; k < pieces; k += 32) M = fmaxf(M, __ldcg(a.part_ml + slot(k)).x);
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, s));
        float acc[PER], l = 0.f;
#pragma unroll
        for (int u = 0; u < PER; ++u) acc[u] = 0.f;
#pragma unroll 4
        for (int k = 0; k < pieces; ++k) {
            const float2 ml = __ldcg(a.part_ml + slot(k));
            const float* const o = a.part_o + slot(k) * D + PER * lane;
            float v[PER];
            if constexpr (PER == 4) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(o));
                v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
            } else {
                const float2 t = __ldcg(reinterpret_cast<const float2*>(o));
                v[0] = t.x; v[1] = t.y;
            }
            if (ml.x == -INFINITY && ml.y == 0.f) continue;             // the row saw none of this part
            const float w = ml.x == M ? 1.f : exp2f((ml.x - M) * a.unit);
            l = fmaf(ml.y, w, l);
#pragma unroll
            for (int u = 0; u < PER; ++u) acc[u] = fmaf(v[u], w, acc[u]);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16* const to = a.out + ((int64_t)(d.y + (r >> a.g_shift)) * a.Hq + d.w * G + (r & (G - 1))) * D + PER * lane;
        if constexpr (PER == 4)
            *reinterpret_cast<uint2*>(to) = make_uint2(pf_pack(acc[0] * inv, acc[1] * inv), pf_pack(acc[2] * inv, acc[3] * inv));
        else
            *reinterpret_cast<uint32_t*>(to) = pf_pack(acc[0] * inv, acc[1] * inv);
    }
}

// ------------------------------------------------------------------------------------------------ host

struct PfScratch { size_t desc, part_ml, part_o, total; };
static PfScratch pf_scratch(int D) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    PfScratch s;
    s.desc = 0;
    s.part_ml = up(sizeof(int4) * PF_MAX_CTAS);
    s.part_o = up(s.part_ml + sizeof(float2) * 2 * PF_MAX_CTAS * PF_ROWS);
    s.total = up(s.part_o + sizeof(float) * 2 * PF_MAX_CTAS * PF_ROWS * D);
    return s;
}

static int pf_validate(const eta_cache_desc* d) {
    int rc = validate_shape(d);
    if (rc == ETA_OK) rc = validate_strides(d);
    if (rc != ETA_OK) return rc;
    return d->batch > PF_MAX_BATCH || d->n_kv_heads > 1024 ? ETA_ERR_UNSUPPORTED : ETA_OK;
}

template <int D, bool GATED>
static int pf_launch(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PrefillArgs& a, int ctas, cudaStream_t s) {
    // the warps' shares of the registers are drawn from what the block is launched with
    cudaFuncAttributes attr;
    const cudaError_t e = cudaFuncGetAttributes(&attr, prefill_kernel<D, GATED>);
    if (e != cudaSuccess) { set_cuda_error(e, "eta_prefill"); return ETA_ERR_CUDA; }
    if (attr.numRegs < PF_REGS) return ETA_ERR_UNSUPPORTED;
    const int rc = launch_pdl("eta_prefill", prefill_kernel<D, GATED>, dim3(ctas), dim3(PF_THREADS), PfSmem<D>::BYTES, s, tmQ, tmK, tmV, a);
    if (rc != ETA_OK) return rc;
    if (a.t_cap <= PF_WHOLE_TOKENS) return ETA_OK;         // nothing to join
    return launch_pdl("eta_prefill", prefill_join_kernel<D>, dim3(ctas, PF_ROWS / PF_JOIN_ROWS), dim3(32 * PF_JOIN_WARPS), 0, s, a);
}

template <int ITEM_COST>
static int check_shares(int batch, int n_kv_heads, int g_shift, int head_dim, int ctas, const int32_t* n, const int32_t* len, int* whole) {
    static thread_local PfTables tab;
    const int m = PF_ROWS >> g_shift;
    tab.longest = 0;
    tab.items[0] = 0; tab.cost[0] = 0;
    int rows = 0, longest = 0;             // the longest sequence, the least t_cap
    for (int i = 0; i < batch; ++i) {
        longest = std::max(longest, len[i]);
        const PfTiles<ITEM_COST> ti(len[i], n[i], m);
        tab.row0[i] = rows; tab.n[i] = n[i]; tab.len[i] = len[i];
        rows += n[i];
        tab.items[i + 1] = tab.items[i] + ti.nq * n_kv_heads;
        tab.cost[i + 1] = tab.cost[i] + n_kv_heads * ti.cost_before(ti.nq);
        int64_t sum = 0;
        for (int t = 0; t < ti.nq; ++t) {
            if (ti.cost_before(t) != sum) return 1;
            tab.longest = std::max(tab.longest, ti.weight(t) * ti.tiles(t));
            sum += (int64_t)ti.weight(t) * ti.tiles(t) + ITEM_COST;
        }
        if (ti.cost_before(ti.nq) != sum) return 2;
    }
    // per item: next tile expected, parts seen, parts announced
    struct Seen { int next = 0, parts = 0, said = 0, last = -2; };
    std::vector<Seen> seen((size_t)rows * n_kv_heads + 1);
    for (int c = 0; c < ctas; ++c) {
        PfWalk<ITEM_COST> w(tab, batch, n_kv_heads, g_shift, head_dim, c, ctas);
        *whole = w.whole;
        PfItem it;
        int starts = 0;
        while (w.next(it)) {
            if (it.seq < 0 || it.seq >= batch || it.hk < 0 || it.hk >= n_kv_heads || it.n_tok < 1 || it.n_tok > m) return 3;
            const int tok = it.row0 - tab.row0[it.seq];
            if (tok < 0 || tok % m || tok + it.n_tok > n[it.seq] || it.p0 != len[it.seq] - n[it.seq] + tok) return 4;
            Seen& s = seen[(size_t)it.row0 * n_kv_heads + it.hk];
            const int all = it.p0 + it.n_tok > 0 ? (it.p0 + it.n_tok - 1) / PF_TILE + 1 : 0, got = std::max(0, it.k1 - it.k0);
            if (it.twin ? it.n0 + it.n1 != got || 2 * it.n_tok > m : (2 * it.n_tok > m ? it.n1 : it.n0) != got) return 11;
            if (it.slot < 0) {
                if (s.parts || it.k0 != 0 || got != all) return 5;
                s.parts = s.said = 1; s.next = all;
                continue;
            }
            if (it.slot != 2 * c && it.slot != 2 * c + 1) return 6;
            if (longest <= PF_WHOLE_TOKENS || !got) return 12;
            if (it.slot == 2 * c + 1) {
                if (it.k0 != 0 || s.parts || ++starts > 1 || it.pieces < 2 || c + it.pieces > ctas) return 7;
                s.said = it.pieces;
            } else if (!s.parts || it.k0 != s.next || s.last != c - 1) {
                return 8;
            }
            s.next = it.k1;
            s.last = c;
            ++s.parts;
        }
    }
    for (int i = 0; i < batch; ++i)
        for (int t = 0; t < n[i]; t += m)
            for (int h = 0; h < n_kv_heads; ++h) {
                const Seen& s = seen[(size_t)(tab.row0[i] + t) * n_kv_heads + h];
                const int end = len[i] - n[i] + std::min(t + m, n[i]), all = end > 0 ? (end - 1) / PF_TILE + 1 : 0;
                if (!s.parts || s.parts != s.said || s.next != all) return 10;
            }
    return 0;
}

}  // namespace eta

extern "C" {

// Host-only check of how work is shared out: for made-up lengths every tile of every item is in exactly one share, the parts of a split
// item have slots of their own, in order, and whoever has the first part knows their number.  Not part of the public interface; called by the
// CPU test-suite.  Where the second kernel is not launched, no item is split.  n, len: [batch] new tokens and tokens cached.  -> 0, the number of the first expectation that failed, or -1: not a problem that
// it can take.
int eta_selftest_prefill_shares(int batch, int n_kv_heads, int g_shift, int head_dim, int ctas, const int32_t* n, const int32_t* len,
                                int* whole) {
    if (batch <= 0 || batch > eta::PF_MAX_BATCH || ctas <= 0 || ctas > eta::PF_MAX_CTAS) return -1;
    try {
        int gated_whole;
        const int rc = eta::check_shares<eta::PF_ITEM_COST<true>>(batch, n_kv_heads, g_shift, head_dim, ctas, n, len, &gated_whole);
        return rc ? rc : eta::check_shares<eta::PF_ITEM_COST<false>>(batch, n_kv_heads, g_shift, head_dim, ctas, n, len, whole);
    } catch (...) {                        // no memory for what it keeps per item
        return -1;
    }
}

int eta_prefill_workspace_bytes(const eta_cache_desc* desc, size_t* out_bytes) {
    if (!out_bytes) return ETA_ERR_INVALID_ARG;
    const int rc = eta::pf_validate(desc);
    if (rc != ETA_OK) return rc;
    *out_bytes = eta::pf_scratch(desc->head_dim).total;
    return ETA_OK;
}

int eta_prefill(const eta_cache_desc* desc, const eta_page_table* pages, const eta_params* params, int32_t n_rows, const void* q,
                const int32_t* row_start, const int32_t* seq_lens, const int32_t* granted, const void* K, const void* V, const float* tau,
                const float* head_const, void* out, uint32_t* status_dev, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace eta;
    int rc = pf_validate(desc);
    if (rc != ETA_OK) return rc;
    if (pages && (rc = validate_pages(desc, pages)) != ETA_OK) return rc;
    if (!params || n_rows < 0 || !row_start || !seq_lens || !K || !V || (n_rows && (!q || !out))) return ETA_ERR_INVALID_ARG;
    const bool dense = (params->flags & ETA_FLAG_DENSE) != 0;
    if (!dense && (tau != nullptr) == (head_const != nullptr)) return ETA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15)
        return ETA_ERR_UNSUPPORTED;
    const int D = desc->head_dim, G = desc->n_q_heads / desc->n_kv_heads;
    // items are counted in 32 bits
    if (n_rows > (1 << 30) || ((int64_t)n_rows * G / PF_ROWS + desc->batch) * desc->n_kv_heads > (1 << 30)) return ETA_ERR_UNSUPPORTED;
    const PfScratch L = pf_scratch(D);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < L.total) return ETA_ERR_WORKSPACE;
    if (n_rows == 0) return ETA_OK;

    const int n_pages = pages ? pages->n_pages : 0;
    CUtensorMap tmQ, tmK, tmV;
    {
        const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)desc->n_q_heads, (cuuint64_t)n_rows};
        const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)desc->n_q_heads * D * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)(PF_HALF / G)};
        if ((rc = encode_tiles(&tmQ, q, 3, dims, strides, box)) != ETA_OK) return rc;
    }
    auto cache_map = [&](CUtensorMap* tm, const void* base, int64_t sb, int64_t sh, int64_t st) {
        const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)(pages ? desc->block_size : desc->t_cap), (cuuint64_t)desc->n_kv_heads,
                                    (cuuint64_t)(pages ? n_pages : desc->batch)};
        const cuuint64_t strides[3] = {(cuuint64_t)st * 2, (cuuint64_t)sh * 2, (cuuint64_t)sb * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)(pages ? desc->block_size : PF_TILE), 1, 1};
        return encode_tiles(tm, base, 4, dims, strides, box);
    };
    if ((rc = cache_map(&tmK, K, desc->k_stride_b, desc->k_stride_h, desc->k_stride_t)) != ETA_OK) return rc;
    if ((rc = cache_map(&tmV, V, desc->v_stride_b, desc->v_stride_h, desc->v_stride_t)) != ETA_OK) return rc;

    int dev = 0, n_sm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) { set_cuda_error(e, "device query"); return ETA_ERR_CUDA; }
    const int ctas = n_sm < PF_MAX_CTAS ? n_sm : PF_MAX_CTAS;

    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    PrefillArgs a;
    a.row_start = row_start; a.seq_lens = seq_lens; a.granted = granted;
    a.block_table = pages ? pages->block_table : nullptr;
    a.table_stride = pages ? pages->table_stride : 0;
    a.n_pages = n_pages;
    a.tau = tau; a.head_const = head_const;
    a.V = static_cast<const __nv_bfloat16*>(V);
    a.v_sb = desc->v_stride_b; a.v_sh = desc->v_stride_h; a.v_st = desc->v_stride_t;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.desc = reinterpret_cast<int4*>(ws + L.desc);
    a.part_ml = reinterpret_cast<float2*>(ws + L.part_ml);
    a.part_o = reinterpret_cast<float*>(ws + L.part_o);
    a.status = status_dev;
    a.a = params->a; a.beta = params->beta;
    a.scale = params->scale > 0.f ? params->scale : 1.0f / sqrtf((float)D);
    a.batch = desc->batch; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads;
    a.g_shift = G == 1 ? 0 : (G == 2 ? 1 : (G == 4 ? 2 : 3));
    a.b_shift = desc->block_size == 32 ? 5 : (desc->block_size == 64 ? 6 : 7);
    a.t_cap = desc->t_cap; a.n_rows = n_rows;
    a.unit = dense ? a.scale * 1.4426950408889634f : 1.f;
    a.ungate = (params->flags & ETA_FLAG_UNGATE_LAST) ? 1 : 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (D == 128) return dense ? pf_launch<128, false>(tmQ, tmK, tmV, a, ctas, s) : pf_launch<128, true>(tmQ, tmK, tmV, a, ctas, s);
    return dense ? pf_launch<64, false>(tmQ, tmK, tmV, a, ctas, s) : pf_launch<64, true>(tmQ, tmK, tmV, a, ctas, s);
}

}  // extern "C"
