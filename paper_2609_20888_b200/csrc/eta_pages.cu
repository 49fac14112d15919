// Pages of a cache that several sequences hold: forks, the release of what nobody holds any more, compaction, and the copies that
// these ask for.  A page that n sequences hold has shared[page] = n - 1; only full pages are shared, since nobody writes to them again.
//
// What these wait for is latency: a few thousand page numbers in dependent steps.  fork, free and compact are one launch each: a CTA
// where there is little to do, else a cluster of eight, whose barriers part the steps (a kernel per step is 2 us more for each).  Page
// numbers travel through memory (the L2); what depends on an order is a prefix sum over the sequences (fork) or over a bit per page
// (free, compact), so results do not depend on how the atomics fall: free pages go onto the stack by number, moves are in pairs by number.
#include "eta_common.cuh"

namespace eta {

constexpr int PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32, PG_CLUSTER = 8;
constexpr int PG_MAX_BATCH = 1024;         // of a fork: a sequence per thread
constexpr int PG_CHUNK = 128;              // pages of a sequence that a warp takes at a time
// Entries (pages and table) up to which one CTA does it.  One CTA against a cluster, us in a row of calls, for forks, releases and compaction: at 2.7K
// entries 3.9 / 4.6, 4.2 / 7.0, 6.3 / 9.8; at 5.5K 5.0 / 5.8, 5.3 / 8.1, 8.3 / 10.5; at 11K 7.3 / 6.5, 6.9 / 8.3, 11.8 / 10.3; at 22K 11.8 / 6.6,
// 10.5 / 8.6, 20.7 / 11.5.
constexpr int64_t PG_SMALL = 4096;

template <int N>
__device__ __forceinline__ void pg_sync() {
    if constexpr (N == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

// The sum of x over the threads before this one; all: over all.  s_warp may be used again after the next barrier.
__device__ __forceinline__ int pg_scan(int x, int& all, int* s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int u = x;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, u, s);
        if (lane >= s) u += o;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = u;
    __syncthreads();
    int w = s_warp[lane];
    const int mine = w;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, w, s);
        if (lane >= s) w += o;
    }
    all = __shfl_sync(0xffffffffu, w, 31);
    return __shfl_sync(0xffffffffu, w - mine, warp) + u - x;
}
static_assert(PG_WARPS == 32, "a lane per warp");

struct PagesArgs {
    int batch, b_shift, t_cap, most, stride, n_pages;  // most: pages that a sequence can have
    const int32_t *seq_lens, *table, *shared, *n_free;
    int32_t *seq_lens_out, *table_out, *shared_out, *free_pages, *n_free_out;
    uint32_t *bits, *status;                           // scratch: a bit per page
    int32_t *before, *count;                           // scratch: free pages before a word's; per CTA
    // free
    const int32_t* release;
    // fork
    const int32_t *parent, *take;
    int32_t *copy_src, *copy_dst, *granted;
    // compact
    const int32_t* free_in;
    int32_t *to, *move_src, *move_dst, *n_moves;       // to: scratch, where a page goes
};

__device__ __forceinline__ int pg_clamped(int n, int most) { return n < 0 ? 0 : (n > most ? most : n); }
// pages that a sequence of n tokens holds
__device__ __forceinline__ int pg_held(int n, const PagesArgs& a) {
    return n <= 0 ? 0 : min(a.most, (int)(((int64_t)n + (1 << a.b_shift) - 1) >> a.b_shift));
}
__device__ __forceinline__ void pg_refuse(bool refused, const PagesArgs& a) {
    if (__any_sync(0xffffffffu, refused) && (threadIdx.x & 31) == 0 && a.status) atomicOr(a.status, ETA_DEV_REFUSED);
}

// Counts as they come out; negative ones count as 0.
template <int NT>
__device__ __forceinline__ void pg_counts(const PagesArgs& a, int tid) {
#pragma unroll 4
    for (int p = tid; p < a.n_pages; p += NT) {
        const int n = __ldcg(a.shared + p);
        if (n < 0 || a.shared_out != a.shared) a.shared_out[p] = max(n, 0);
    }
}

// Free pages by number: word w of the bits belongs to CTA w / per.  f(word's index, its bits, free pages before it).
template <int N, typename F>
__device__ __forceinline__ int pg_bits(const PagesArgs& a, int rank, int* s_warp, F f) {
    const int words = (a.n_pages + 31) / 32, per = (words + N - 1) / N, w0 = min(words, rank * per), w1 = min(words, w0 + per);
    int base = 0, all;
    if constexpr (N > 1) {
        int n = 0;
        for (int w = w0 + (int)threadIdx.x; w < w1; w += PG_THREADS) n += __popc(__ldcg(a.bits + w));
        pg_scan(n, all, s_warp);
        if (threadIdx.x == 0) a.count[rank] = all;
        pg_sync<N>();
        all = 0;
        for (int r = 0; r < N; ++r) {
            const int c = __ldcg(a.count + r);
            base += r < rank ? c : 0;
            all += c;
        }
    } else {
        all = 0;
    }
    for (int w = w0; w < w1; w += PG_THREADS) {
        const int i = w + (int)threadIdx.x;
        const uint32_t v = i < w1 ? __ldcg(a.bits + i) : 0u;
        int here;
        const int at = pg_scan(__popc(v), here, s_warp);
        if (i < w1) f(i, v, base + at);
        base += here;
    }
    return N > 1 ? all : base;
}

// ------------------------------------------------------------------------------------------------ free

template <int N>
__global__ void __launch_bounds__(PG_THREADS) free_pages_kernel(const PagesArgs a) {
    __shared__ int s_warp[PG_WARPS];
    const int rank = N > 1 ? blockIdx.x : 0, tid = rank * PG_THREADS + threadIdx.x, lane = threadIdx.x & 31;
    constexpr int NT = N * PG_THREADS;
    bool refused = false;
    pdl_wait();
    const int n_free = pg_clamped(__ldcg(a.n_free), a.n_pages);
    const int top = tid < n_free ? __ldcg(a.free_pages + tid) : -1;
    for (int w = tid; w < (a.n_pages + 31) / 32; w += NT) a.bits[w] = 0u;
    pg_counts<NT>(a, tid);
    pg_sync<N>();
    // a bit per page on the stack: those that come back must not be among them
    auto mark = [&](int page) {
        if (page >= 0 && page < a.n_pages) atomicOr(a.bits + page / 32, 1u << (page & 31));
    };
    mark(top);
    for (int k = tid + NT; k < n_free; k += NT) mark(__ldcg(a.free_pages + k));
    // Everyone that lets go counts down, without looking: a count that ends below zero has nobody left.  (Looking at what each
    // atomic returns, 800 sequences took 54 us.)
    const int chunks = (a.most + PG_CHUNK - 1) / PG_CHUNK;
    const int64_t units = (int64_t)a.batch * chunks;
    int goes = 0, len = 0;
    auto fetch = [&](int64_t u) {
        if (u >= units) return;
        goes = __ldcg(a.release + u / chunks);
        len = __ldcg(a.seq_lens + u / chunks);
    };
    fetch(tid / 32);
    for (int64_t u = tid / 32; u < units; u += NT / 32) {
        const int i = (int)(u / chunks), j0 = (int)(u % chunks) * PG_CHUNK, held = goes ? pg_held(len, a) : 0;
        fetch(u + NT / 32);
        if (j0 >= held) continue;
        int page[PG_CHUNK / 32];
#pragma unroll
        for (int k = 0; k < PG_CHUNK / 32; ++k) {
            const int j = j0 + 32 * k + lane;
            page[k] = j < held ? __ldcg(a.table + (int64_t)i * a.stride + j) : -1;
            if (j < held && (page[k] < 0 || page[k] >= a.n_pages)) { refused = true; page[k] = -1; }
        }
#pragma unroll
        for (int k = 0; k < PG_CHUNK / 32; ++k)
            if (page[k] >= 0) atomicSub(a.shared_out + page[k], 1);
    }
    pg_sync<N>();
    {
        // a bit per page that comes back, of the words that this CTA goes on with
        const int words = (a.n_pages + 31) / 32, per = (words + N - 1) / N, w1 = min(words, (rank + 1) * per);
        for (int w = rank * per + (int)threadIdx.x / 32; w < w1; w += PG_WARPS) {
            const int p = 32 * w + lane, n = p < a.n_pages ? __ldcg(a.shared_out + p) : 0;
            const uint32_t stack = __ldcg(a.bits + w);
            if (n < 0) a.shared_out[p] = 0;
            refused = refused || n < -1 || (n < 0 && ((stack >> lane) & 1u));
            const uint32_t v = __ballot_sync(0xffffffffu, n < 0) & ~stack;
            if (lane == 0) a.bits[w] = v;
        }
        __syncthreads();
    }
    const int back = pg_bits<N>(a, rank, s_warp, [&](int w, uint32_t v, int at) {
        for (; v; v &= v - 1, ++at) {
            const int page = 32 * w + __ffs(v) - 1;
            if (n_free + at < a.n_pages) a.free_pages[n_free + at] = page;
            else refused = true;
        }
    });
    for (int i = tid; i < a.batch; i += NT) {
        const int n = __ldcg(a.seq_lens + i);
        if (__ldcg(a.release + i)) a.seq_lens_out[i] = 0;
        else if (a.seq_lens_out != a.seq_lens) a.seq_lens_out[i] = n;
    }
    if (tid == 0) *a.n_free_out = min(a.n_pages, n_free + back);
    pg_refuse(refused, a);
}

// ------------------------------------------------------------------------------------------------ fork

template <int N>
__global__ void __launch_bounds__(PG_THREADS) fork_pages_kernel(const PagesArgs a) {
    __shared__ int s_warp[PG_WARPS], s_parent[PG_MAX_BATCH], s_whole[PG_MAX_BATCH];      // whole: pages shared
    const int rank = N > 1 ? blockIdx.x : 0, tid = rank * PG_THREADS + threadIdx.x, lane = threadIdx.x & 31, i = threadIdx.x;
    constexpr int NT = N * PG_THREADS;
    bool refused = false;
    pdl_wait();
    const int n_free = pg_clamped(__ldcg(a.n_free), a.n_pages);
    int u = -1, T = 0, mine = 0;
    if (i < a.batch) {
        u = __ldcg(a.parent + i);
        mine = __ldcg(a.seq_lens + i);
        if (u >= 0) {
            // a parent is a sequence of its own, and the child's place is empty
            const bool fits = u < a.batch && u != i && mine <= 0 && __ldcg(a.parent + u) < 0;
            if (fits) {
                T = pg_clamped(__ldcg(a.seq_lens + u), a.t_cap);
                if (a.take) T = min(T, max(__ldcg(a.take + i), 0));
            } else {
                refused = true;
                u = -1;
            }
        }
    }
    // Both pages of a copy have to be ones: the parent's last, before the child counts as one that wants a page, and the one off the stack.
    auto is_page = [&](int page) { return page >= 0 && page < a.n_pages; };
    const int whole = T >> a.b_shift;
    int tail = (T & ((1 << a.b_shift) - 1)) != 0, src = -1, dst = -1;
    if (tail) {
        src = __ldcg(a.table + (int64_t)u * a.stride + whole);
        if (!is_page(src)) { refused = true; u = -1; tail = 0; }
    }
    int wanted;
    const int nth = pg_scan(tail, wanted, s_warp);
    bool ok = u >= 0 && (!tail || nth < n_free);
    if (ok && tail) {
        dst = __ldcg(a.free_pages + n_free - 1 - nth);
        ok = is_page(dst);
    }
    refused = refused || (u >= 0 && !ok);
    s_parent[i] = u;
    s_whole[i] = ok ? whole : 0;
    const bool copies = ok && tail;
    pg_counts<NT>(a, tid);
    pg_sync<N>();          // all is read that may be written in place
    if (rank == 0 && i < a.batch) {
        a.granted[i] = ok ? T : 0;
        a.copy_src[i] = copies ? src : -1;
        a.copy_dst[i] = copies ? dst : -1;
        if (copies) a.table_out[(int64_t)i * a.stride + whole] = dst;
        if (ok) a.seq_lens_out[i] = T;
        else if (a.seq_lens_out != a.seq_lens) a.seq_lens_out[i] = mine;
        if (i == 0) *a.n_free_out = n_free - min(wanted, n_free);
    }
    if (rank == 0) pg_refuse(refused, a);
    bool bad = false;
    const int chunks = (a.most + PG_CHUNK - 1) / PG_CHUNK;
    for (int64_t c = tid / 32; c < (int64_t)a.batch * chunks; c += NT / 32) {
        const int child = (int)(c / chunks), j0 = (int)(c % chunks) * PG_CHUNK, n = s_whole[child];
        if (j0 >= n) continue;
        const int32_t* const from = a.table + (int64_t)s_parent[child] * a.stride;
        int32_t* const to = a.table_out + (int64_t)child * a.stride;
        int page[PG_CHUNK / 32];
#pragma unroll
        for (int k = 0; k < PG_CHUNK / 32; ++k) page[k] = j0 + 32 * k + lane < n ? __ldcg(from + j0 + 32 * k + lane) : -1;
#pragma unroll
        for (int k = 0; k < PG_CHUNK / 32; ++k) {
            const int j = j0 + 32 * k + lane;
            if (j >= n) continue;
            to[j] = page[k];
            if (page[k] >= 0 && page[k] < a.n_pages) atomicAdd(a.shared_out + page[k], 1);
            else bad = true;
        }
    }
    pg_refuse(bad, a);
}

// ------------------------------------------------------------------------------------------------ compact

template <int N>
__global__ void __launch_bounds__(PG_THREADS) compact_pages_kernel(const PagesArgs a) {
    __shared__ int s_warp[PG_WARPS];
    const int rank = N > 1 ? blockIdx.x : 0, tid = rank * PG_THREADS + threadIdx.x;
    constexpr int NT = N * PG_THREADS;
    bool refused = false;
    pdl_wait();
    const int said = __ldcg(a.n_free), n_free = pg_clamped(said, a.n_pages);
    const int words = (a.n_pages + 31) / 32;
    for (int w = tid; w < words; w += NT) a.bits[w] = 0u;
    pg_sync<N>();
    for (int k = tid; k < n_free; k += NT) {
        const int page = __ldcg(a.free_in + k);
        if (page >= 0 && page < a.n_pages) atomicOr(a.bits + page / 32, 1u << (page & 31));
        else refused = true;
    }
    pg_sync<N>();
    const int F = pg_bits<N>(a, rank, s_warp, [&](int w, uint32_t, int at) { a.before[w] = at; });
    const int live = a.n_pages - F;
    refused = refused || F != said;
    pg_sync<N>();
    // free pages before page p (p <= n_pages)
    auto free_before = [&](int p) {
        return p == a.n_pages ? F : __ldcg(a.before + p / 32) + __popc(__ldcg(a.bits + p / 32) & ((1u << (p & 31)) - 1u));
    };
    auto is_free = [&](int p) { return (__ldcg(a.bits + p / 32) >> (p & 31)) & 1u; };
    const int moves = free_before(live);                // free pages below the line, as many as live ones above it
    for (int p = tid; p < a.n_pages; p += NT) {
        const bool f = is_free(p);
        if (p < live ? f : !f) {
            const int k = p < live ? free_before(p) : p - live - (free_before(p) - moves);
            (p < live ? a.move_dst : a.move_src)[k] = p;
        } else if (a.shared_out != a.shared) {
            a.shared_out[p] = max(__ldcg(a.shared + p), 0);
        }
    }
    pg_sync<N>();
    for (int k = tid; k < moves; k += NT) {
        const int src = __ldcg(a.move_src + k), dst = __ldcg(a.move_dst + k), held = max(__ldcg(a.shared + src), 0);
        a.to[src] = dst;
        a.shared_out[dst] = held;
        a.shared_out[src] = 0;
    }
    // (the stack was read before the second barrier)
    for (int k = tid; k < F; k += NT) a.free_pages[k] = a.n_pages - 1 - k;
    if (tid == 0) { *a.n_moves = moves; *a.n_free_out = F; }
    pg_sync<N>();
    const int64_t entries = (int64_t)a.batch * a.most;
    for (int64_t e = tid; e < entries; e += NT) {
        const int i = (int)(e / a.most), j = (int)(e % a.most);
        const int64_t at = (int64_t)i * a.stride + j;
        int page = __ldcg(a.table + at);
        const int was = page;
        if (j < pg_held(__ldcg(a.seq_lens + i), a)) {
            if (page < 0 || page >= a.n_pages || is_free(page)) refused = true;
            else if (page >= live) page = __ldcg(a.to + page);
        }
        if (page != was || a.table_out != a.table) a.table_out[at] = page;
    }
    pg_refuse(refused, a);
}

// ------------------------------------------------------------------------------------------------ copies

constexpr int PC_THREADS = 256, PC_UNROLL = 8, PC_BYTES = 16 * PC_THREADS * PC_UNROLL;        // bytes that a CTA has under way
constexpr int PC_MAX_POOLS = 64;

// bytes (a multiple of 16, at most PC_BYTES) from one place to another, all loads before the first store
__device__ __forceinline__ void pc_copy(unsigned char* to, const unsigned char* from, int bytes) {
    uint4 v[PC_UNROLL];
#pragma unroll
    for (int u = 0; u < PC_UNROLL; ++u) {
        const int at = 16 * ((int)threadIdx.x + u * PC_THREADS);
        if (at < bytes) v[u] = __ldcg(reinterpret_cast<const uint4*>(from + at));
    }
#pragma unroll
    for (int u = 0; u < PC_UNROLL; ++u) {
        const int at = 16 * ((int)threadIdx.x + u * PC_THREADS);
        if (at < bytes) *reinterpret_cast<uint4*>(to + at) = v[u];
    }
}

struct CopyArgs {
    eta_page_pool pool[PC_MAX_POOLS];
    int32_t first[PC_MAX_POOLS + 1];                   // pieces of PC_BYTES of a page before a pool's
    int n_pools, n_pages, max_moves;
    const int32_t *src, *dst, *n_moves;
    uint32_t* status;
};

// A page of all pools is cut into pieces of 32 KB, which the CTAs take in turns.  Bound by memory: some
// 371 MB (read and written) in 60 us, 6.2 TB/s.  Other numbers of CTAs, threads and loads under way: moves 83 to 89 us in all instead of 85, forks 148
// to 167 instead of 144; with streaming hints 93 and 205.
__global__ void __launch_bounds__(PC_THREADS) copy_pages_kernel(const __grid_constant__ CopyArgs a) {
    pdl_wait();
    const int n = a.n_moves ? pg_clamped(__ldcg(a.n_moves), a.max_moves) : a.max_moves, per = a.first[a.n_pools];
    for (int64_t u = blockIdx.x; u < (int64_t)n * per; u += gridDim.x) {
        const int k = (int)(u / per), piece = (int)(u % per);
        const int src = __ldcg(a.src + k), dst = __ldcg(a.dst + k);
        if (src < 0 || dst < 0) continue;
        if (src >= a.n_pages || dst >= a.n_pages) {
            if (threadIdx.x == 0 && a.status) atomicOr(a.status, ETA_DEV_BAD_SLOT);
            continue;
        }
        int q = 0;
        while (piece >= a.first[q + 1]) ++q;
        const eta_page_pool& pool = a.pool[q];
        const int cut = (int)((pool.piece_bytes + PC_BYTES - 1) / PC_BYTES), at = piece - a.first[q], row = at / cut;
        const int64_t off = (int64_t)(at % cut) * PC_BYTES;
        unsigned char* const base = static_cast<unsigned char*>(pool.base) + (int64_t)row * pool.piece_stride + off;
        pc_copy(base + (int64_t)dst * pool.page_stride, base + (int64_t)src * pool.page_stride, (int)min((int64_t)PC_BYTES, pool.piece_bytes - off));
    }
}

struct ForkSummaryArgs {
    const int32_t *parent, *granted;
    unsigned char* musig;
    float* mnorm;
    uint32_t* status;
    int batch, Hkv, nb_cap, record, b_shift;
};

// Records of a child's full blocks, one run per KV head.  What a CTA takes is found in the prefix sums over the children, which it
// makes for itself.
constexpr int FS_PER = PG_MAX_BATCH / PC_THREADS;
__global__ void __launch_bounds__(PC_THREADS) fork_summaries_kernel(const ForkSummaryArgs a) {
    __shared__ int s_before[PG_MAX_BATCH + 1], s_warp[PC_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    const int per_piece = PC_BYTES / a.record;          // records of a piece
    int n[FS_PER], sum = 0;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < FS_PER; ++k) {
        const int i = tid * FS_PER + k;
        n[k] = 0;
        if (i < a.batch) {
            const int u = __ldcg(a.parent + i);
            if (u >= 0) {
                const int nb = min(max(__ldcg(a.granted + i), 0) >> a.b_shift, a.nb_cap);
                if (u >= a.batch || u == i) bad = bad || nb > 0;
                else n[k] = (nb + per_piece - 1) / per_piece * a.Hkv;
            }
        }
        sum += n[k];
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0 && blockIdx.x == 0 && a.status) atomicOr(a.status, ETA_DEV_REFUSED);
    int x = sum;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, x, s);
        if (lane >= s) x += o;
    }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    x -= sum;
    for (int w = 0; w < warp; ++w) x += s_warp[w];
#pragma unroll
    for (int k = 0; k < FS_PER; ++k) {
        s_before[tid * FS_PER + k] = x;
        x += n[k];
    }
    if (tid == PC_THREADS - 1) s_before[PG_MAX_BATCH] = x;
    __syncthreads();
    const int all = s_before[PG_MAX_BATCH];
    for (int p = blockIdx.x; p < all; p += gridDim.x) {
        int lo = 0, hi = PG_MAX_BATCH;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_before[mid] <= p) lo = mid; else hi = mid;
        }
        const int i = lo, u = __ldcg(a.parent + i), nb = min(__ldcg(a.granted + i) >> a.b_shift, a.nb_cap);
        const int cut = (nb + per_piece - 1) / per_piece, at = p - s_before[i], hk = at / cut, j0 = (at % cut) * per_piece, m = min(per_piece, nb - j0);
        const int64_t to = ((int64_t)i * a.Hkv + hk) * a.nb_cap + j0, from = ((int64_t)u * a.Hkv + hk) * a.nb_cap + j0;
        for (int j = tid; j < m; j += PC_THREADS) a.mnorm[to + j] = __ldcg(a.mnorm + from + j);
        pc_copy(a.musig + to * a.record, a.musig + from * a.record, m * a.record);
    }
}

// ------------------------------------------------------------------------------------------------ host

struct PagesScratch { size_t before, to, count, total; };
static PagesScratch pages_scratch(int32_t n_pages) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t words = up(4 * (((size_t)n_pages + 31) / 32));
    PagesScratch s;
    s.before = words;
    s.to = 2 * words;
    s.count = s.to + up(4 * (size_t)n_pages);
    s.total = s.count + 256;
    return s;
}
static int pages_check(int32_t batch, int32_t block_size, int32_t t_cap, int32_t table_stride, int32_t n_pages) {
    if (batch <= 0 || t_cap <= 0 || table_stride <= 0 || n_pages <= 0) return ETA_ERR_INVALID_ARG;
    if (block_size != 32 && block_size != 64 && block_size != 128) return ETA_ERR_UNSUPPORTED;
    if ((int64_t)table_stride * block_size < t_cap) return ETA_ERR_INVALID_ARG;
    return batch > (1 << 30) || n_pages > (1 << 30) ? ETA_ERR_UNSUPPORTED : ETA_OK;
}
static PagesArgs pages_args(int32_t batch, int32_t block_size, int32_t t_cap, int32_t table_stride, int32_t n_pages, uint32_t* status) {
    PagesArgs a = {};
    a.batch = batch; a.b_shift = block_size == 32 ? 5 : (block_size == 64 ? 6 : 7);
    a.most = (int)(((int64_t)t_cap + block_size - 1) / block_size);
    a.t_cap = t_cap; a.stride = table_stride; a.n_pages = n_pages; a.status = status;
    return a;
}
static int pages_workspace(PagesArgs& a, void* workspace, size_t bytes) {
    const PagesScratch s = pages_scratch(a.n_pages);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || bytes < s.total) return ETA_ERR_WORKSPACE;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    a.bits = reinterpret_cast<uint32_t*>(ws);
    a.before = reinterpret_cast<int32_t*>(ws + s.before);
    a.to = reinterpret_cast<int32_t*>(ws + s.to);
    a.count = reinterpret_cast<int32_t*>(ws + s.count);
    return ETA_OK;
}
static bool pages_one_cta(int64_t entries, int clusters) {
#ifdef ETA_TEST_GENERAL_PATH
    clusters = 0;
#endif
    return entries <= PG_SMALL || clusters < 1;
}
static int pages_launch(const char* what, void (*one)(PagesArgs), void (*cluster)(PagesArgs), const PagesArgs& a, void* stream) {
    // a part of a GPU may hold no cluster of this size: one CTA does any size then, if slowly
    const int64_t entries = (int64_t)a.batch * a.most + a.n_pages;
    int fit[MAX_CLUSTER + 1] = {};
    if (entries > PG_SMALL) clusters_that_fit(reinterpret_cast<const void*>(cluster), PG_THREADS, 0, fit);
    const bool small = pages_one_cta(entries, fit[PG_CLUSTER]);
    const void* const kernel = reinterpret_cast<const void*>(small ? one : cluster);
    const int rc = configure_kernel(kernel, 0);
    if (rc != ETA_OK) return rc;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = cluster_config(small ? 1 : PG_CLUSTER, 1, PG_THREADS, 0, attr);
    cfg.stream = static_cast<cudaStream_t>(stream);
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, small ? one : cluster, a);
    if (e != cudaSuccess) { set_cuda_error(e, what); return ETA_ERR_CUDA; }
    return check_launch(what);
}
// CTAs that move bytes: enough to have the memory busy
static int copy_ctas(int64_t pieces) {
    int dev = 0, n_sm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) { set_cuda_error(e, "device query"); return ETA_ERR_CUDA; }
    const int64_t most = 4ll * n_sm;
    return (int)(pieces < 1 ? 1 : (pieces < most ? pieces : most));
}

}  // namespace eta

extern "C" {

int eta_pages_workspace_bytes(int32_t n_pages, size_t* out_bytes) {
    if (!out_bytes || n_pages <= 0) return ETA_ERR_INVALID_ARG;
    if (n_pages > (1 << 30)) return ETA_ERR_UNSUPPORTED;
    *out_bytes = eta::pages_scratch(n_pages).total;
    return ETA_OK;
}

// Host-only check of how the calls on pages are launched: one CTA where there is little to do or where no cluster fits.  Not part of the public
// interface; called by the CPU test-suite.  -> 1: one CTA, 0: a cluster.
int eta_selftest_pages_one_cta(int64_t entries, int clusters) { return eta::pages_one_cta(entries, clusters); }

int eta_free_pages(int32_t batch, int32_t block_size, int32_t t_cap, const int32_t* release, const int32_t* seq_lens, int32_t* seq_lens_out,
                   const int32_t* block_table, int32_t table_stride, const int32_t* shared, int32_t* shared_out, int32_t* free_pages,
                   const int32_t* n_free, int32_t* n_free_out, int32_t n_pages, uint32_t* status_dev, void* workspace, size_t workspace_bytes,
                   void* stream) {
    using namespace eta;
    int rc = pages_check(batch, block_size, t_cap, table_stride, n_pages);
    if (rc != ETA_OK) return rc;
    if (!release || !seq_lens || !seq_lens_out || !block_table || !shared || !shared_out || !free_pages || !n_free || !n_free_out)
        return ETA_ERR_INVALID_ARG;
    PagesArgs a = pages_args(batch, block_size, t_cap, table_stride, n_pages, status_dev);
    if ((rc = pages_workspace(a, workspace, workspace_bytes)) != ETA_OK) return rc;
    a.release = release; a.seq_lens = seq_lens; a.seq_lens_out = seq_lens_out; a.table = block_table;
    a.shared = shared; a.shared_out = shared_out; a.free_pages = free_pages; a.n_free = n_free; a.n_free_out = n_free_out;
    return pages_launch("eta_free_pages", free_pages_kernel<1>, free_pages_kernel<PG_CLUSTER>, a, stream);
}

int eta_fork_pages(int32_t batch, int32_t block_size, int32_t t_cap, const int32_t* parent, const int32_t* take, const int32_t* seq_lens,
                   int32_t* seq_lens_out, int32_t* block_table, int32_t table_stride, const int32_t* shared, int32_t* shared_out,
                   const int32_t* free_pages, const int32_t* n_free, int32_t* n_free_out, int32_t n_pages, int32_t* copy_src, int32_t* copy_dst,
                   int32_t* granted, uint32_t* status_dev, void* stream) {
    using namespace eta;
    const int rc = pages_check(batch, block_size, t_cap, table_stride, n_pages);
    if (rc != ETA_OK) return rc;
    if (!parent || !seq_lens || !seq_lens_out || !block_table || !shared || !shared_out || !free_pages || !n_free || !n_free_out || !copy_src ||
        !copy_dst || !granted)
        return ETA_ERR_INVALID_ARG;
    if (batch > PG_MAX_BATCH) return ETA_ERR_UNSUPPORTED;
    PagesArgs a = pages_args(batch, block_size, t_cap, table_stride, n_pages, status_dev);
    a.parent = parent; a.take = take; a.seq_lens = seq_lens; a.seq_lens_out = seq_lens_out; a.table = block_table; a.table_out = block_table;
    a.shared = shared; a.shared_out = shared_out; a.free_pages = const_cast<int32_t*>(free_pages); a.n_free = n_free; a.n_free_out = n_free_out;
    a.copy_src = copy_src; a.copy_dst = copy_dst; a.granted = granted;
    return pages_launch("eta_fork_pages", fork_pages_kernel<1>, fork_pages_kernel<PG_CLUSTER>, a, stream);
}

int eta_compact_pages(int32_t batch, int32_t block_size, int32_t t_cap, const int32_t* seq_lens, const int32_t* block_table,
                      int32_t* block_table_out, int32_t table_stride, const int32_t* shared, int32_t* shared_out, const int32_t* free_pages,
                      int32_t* free_pages_out, const int32_t* n_free, int32_t* n_free_out, int32_t n_pages, int32_t* move_src, int32_t* move_dst,
                      int32_t* n_moves, uint32_t* status_dev, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace eta;
    int rc = pages_check(batch, block_size, t_cap, table_stride, n_pages);
    if (rc != ETA_OK) return rc;
    if (!seq_lens || !block_table || !block_table_out || !shared || !shared_out || !free_pages || !free_pages_out || !n_free || !n_free_out ||
        !move_src || !move_dst || !n_moves)
        return ETA_ERR_INVALID_ARG;
    PagesArgs a = pages_args(batch, block_size, t_cap, table_stride, n_pages, status_dev);
    if ((rc = pages_workspace(a, workspace, workspace_bytes)) != ETA_OK) return rc;
    a.seq_lens = seq_lens; a.table = block_table; a.table_out = block_table_out; a.shared = shared; a.shared_out = shared_out;
    a.free_in = free_pages; a.free_pages = free_pages_out; a.n_free = n_free; a.n_free_out = n_free_out;
    a.move_src = move_src; a.move_dst = move_dst; a.n_moves = n_moves;
    return pages_launch("eta_compact_pages", compact_pages_kernel<1>, compact_pages_kernel<PG_CLUSTER>, a, stream);
}

int eta_copy_pages(const eta_page_pool* pools, int32_t n_pools, int32_t n_pages, const int32_t* src, const int32_t* dst, int32_t max_moves,
                   const int32_t* n_moves, uint32_t* status_dev, void* stream) {
    using namespace eta;
    if (!pools || n_pools <= 0 || n_pages <= 0 || max_moves < 0 || (max_moves && (!src || !dst))) return ETA_ERR_INVALID_ARG;
    if (n_pools > PC_MAX_POOLS) return ETA_ERR_UNSUPPORTED;
    CopyArgs a;
    a.n_pools = n_pools; a.n_pages = n_pages; a.max_moves = max_moves; a.src = src; a.dst = dst; a.n_moves = n_moves; a.status = status_dev;
    int64_t first = 0;
    for (int k = 0; k < n_pools; ++k) {
        const eta_page_pool& p = pools[k];
        if (!p.base || p.n_pieces <= 0 || p.piece_bytes <= 0 || p.page_stride <= 0) return ETA_ERR_INVALID_ARG;
        if ((p.page_stride | p.piece_bytes | (p.n_pieces > 1 ? p.piece_stride : 0)) & 15 || reinterpret_cast<uintptr_t>(p.base) & 15) return ETA_ERR_UNSUPPORTED;
        if (p.n_pieces > 1 && p.piece_stride < p.piece_bytes) return ETA_ERR_INVALID_ARG;
        a.pool[k] = p;
        if (p.n_pieces == 1) a.pool[k].piece_stride = 0;
        a.first[k] = (int32_t)first;
        const int64_t cut = (p.piece_bytes + PC_BYTES - 1) / PC_BYTES;
        if (cut > INT32_MAX) return ETA_ERR_UNSUPPORTED;
        first += p.n_pieces * cut;
        if (first > INT32_MAX) return ETA_ERR_UNSUPPORTED;
    }
    a.first[n_pools] = (int32_t)first;
    if (max_moves == 0) return ETA_OK;
    const int ctas = copy_ctas((int64_t)max_moves * first);
    if (ctas < 0) return ctas;
    return launch_pdl("eta_copy_pages", copy_pages_kernel, dim3((unsigned)ctas), dim3(PC_THREADS), 0, static_cast<cudaStream_t>(stream), a);
}

int eta_fork_summaries(const eta_cache_desc* desc, const int32_t* parent, const int32_t* granted, void* musig, float* mnorm, uint32_t flags,
                       uint32_t* status_dev, void* stream) {
    using namespace eta;
    const int rc = validate_shape(desc);
    if (rc != ETA_OK) return rc;
    if (desc->batch > PG_MAX_BATCH || desc->nb_cap >= (1 << 24)) return ETA_ERR_UNSUPPORTED;
    if (!parent || !granted || !musig || !mnorm || flags & ~ETA_BUILD_PACKED_SIGMA) return ETA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(musig) & 15) return ETA_ERR_UNSUPPORTED;
    ForkSummaryArgs a;
    a.parent = parent; a.granted = granted; a.musig = static_cast<unsigned char*>(musig); a.mnorm = mnorm; a.status = status_dev;
    a.batch = desc->batch; a.Hkv = desc->n_kv_heads; a.nb_cap = desc->nb_cap;
    a.record = (flags & ETA_BUILD_PACKED_SIGMA ? 3 : 4) * desc->head_dim;
    a.b_shift = desc->block_size == 32 ? 5 : (desc->block_size == 64 ? 6 : 7);
    const int64_t cut = (desc->nb_cap + PC_BYTES / a.record - 1) / (PC_BYTES / a.record);
    const int ctas = copy_ctas((int64_t)desc->batch * desc->n_kv_heads * cut);
    if (ctas < 0) return ctas;
    return launch_pdl("eta_fork_summaries", fork_summaries_kernel, dim3((unsigned)ctas), dim3(PC_THREADS), 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"
