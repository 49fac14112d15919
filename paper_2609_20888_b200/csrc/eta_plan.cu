// Block tables and slot maps of a paged cache from request lengths: what a serving loop does between two steps, on the GPU, so that
// the step can be captured and the host need not know the lengths.
//
//   released sequences:  their ceil(len / b) pages go on top of the free stack, sequence after sequence
//   new tokens:          need_i = ceil((len_i + new_i) / b) - ceil(len_i / b) pages come off its top, sequence after sequence
//   row r of sequence i: position p = len_i + (r - row_start_i), slot = table[i][p / b] * b + p % b
//
// Everything that depends on an order hangs on three prefix sums over the sequences (rows, pages back, pages needed): plan_kernel
// is one CTA that scans them 1024 sequences at a time, and moves the pages in equal shares of a warp (whose sequences are found in the
// scan by bisection), so that a few long prompts do not leave it to a few threads.  The rows are its work too while they are few; beyond
// that a kernel over all rows follows.  64 requests with a token each take 4.2 us, which is latency; 200 with prompts of up to 9000
// (0.8 M rows, 9 MB written) 17.4 to 17.9, most of it the one CTA that carries 6K pages back and 9K out.
#include "eta_common.cuh"

namespace eta {

struct PlanArgs {
    int batch, b_shift, t_cap, table_stride, n_pages, n_rows;
    const int32_t *new_lens, *release, *seq_lens, *n_free;
    int32_t *seq_lens_out, *n_free_out, *block_table, *free_pages, *positions, *row_start, *granted;
    int64_t* slot_map;
    uint32_t* status;
};

constexpr int PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32;

// The sums of x and y over the threads before this one; all: over all of them.  Every thread of the CTA calls it; s_warp may be used again at
// once (its first half is read before the second barrier only, its second half is written after the next call's first).
__device__ __forceinline__ longlong2 scan(int64_t x, int64_t y, longlong2& all, longlong2* s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t ux = x, uy = y;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int64_t ox = __shfl_up_sync(0xffffffffu, ux, s), oy = __shfl_up_sync(0xffffffffu, uy, s);
        if (lane >= s) { ux += ox; uy += oy; }
    }
    if (lane == 31) s_warp[warp] = make_longlong2(ux, uy);
    __syncthreads();
    if (warp == 0) {
        const longlong2 w = s_warp[lane];
        int64_t wx = w.x, wy = w.y;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t ox = __shfl_up_sync(0xffffffffu, wx, s), oy = __shfl_up_sync(0xffffffffu, wy, s);
            if (lane >= s) { wx += ox; wy += oy; }
        }
        s_warp[PLAN_WARPS + lane] = make_longlong2(wx, wy);
    }
    __syncthreads();
    all = s_warp[2 * PLAN_WARPS - 1];
    const longlong2 before = warp ? s_warp[PLAN_WARPS + warp - 1] : make_longlong2(0, 0);
    return make_longlong2(before.x + ux - x, before.y + uy - y);
}
__device__ __forceinline__ int32_t saturated(int64_t x) { return (int32_t)(x > INT32_MAX ? INT32_MAX : x); }

// the last of n ascending numbers, the first of which is not above x, that is not above x
template <typename At>
__device__ __forceinline__ int last_where_not_above(At at, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at(mid) <= x) lo = mid; else hi = mid;
    }
    return lo;
}
// of numbers in shared memory
__device__ __forceinline__ int last_not_above(const int32_t* v, int n, int32_t x) {
    return last_where_not_above([&](int k) { return v[k]; }, n, x);
}
// of numbers in global memory, which this launch or the one before it wrote
__device__ __forceinline__ int last_not_above_in_memory(const int32_t* v, int n, int32_t x) {
    return last_where_not_above([&](int k) { return __ldcg(v + k); }, n, x);
}

// Pages 0 .. n - 1; s is the last of n_seq ascending numbers that is not above p.  A warp takes consecutive pages, so that it looks for its first
// sequence once and a lane looks again only where its page is past the sequence it is at: with a bisection per page it was the instructions of
// one SM that 200 requests with prompts waited for (21.5 -> 17.5 us).  MOVE loads before the first store, which the compiler would not do, since tables and stack could be the same memory.
constexpr int MOVE = 8;
template <typename Load, typename Store>
__device__ __forceinline__ void move_pages(const int32_t* before, int n_seq, int n, Load load, Store store) {
    const int per_warp = (n + PLAN_THREADS - 1) / PLAN_THREADS * 32, begin = (threadIdx.x >> 5) * per_warp, end = min(n, begin + per_warp);
    if (begin >= end) return;
    int s = last_not_above(before, n_seq, begin), next = s + 1 < n_seq ? before[s + 1] : INT32_MAX;
    for (int p0 = begin + (threadIdx.x & 31); p0 < end; p0 += 32 * MOVE) {
        int of[MOVE], page[MOVE];
#pragma unroll
        for (int u = 0; u < MOVE; ++u) {
            const int p = p0 + 32 * u;
            if (p >= end) continue;
            if (p >= next) {
                s += last_not_above(before + s, n_seq - s, p);
                next = s + 1 < n_seq ? before[s + 1] : INT32_MAX;
            }
            of[u] = s;
            page[u] = load(s, p);
        }
#pragma unroll
        for (int u = 0; u < MOVE; ++u)
            if (p0 + 32 * u < end) store(of[u], p0 + 32 * u, page[u]);
    }
}

// What a row of a sequence needs: position = row + shift; NO_PLACE where the sequence got nothing
constexpr int32_t NO_PLACE = INT32_MIN;
__device__ __forceinline__ int32_t shift_of(int len_after, int got, int row0) { return got > 0 ? len_after - got - row0 : NO_PLACE; }

__device__ __forceinline__ void store_row(const PlanArgs& a, int r, int i, int32_t shift) {
    int64_t slot = -1;
    int pos = 0;
    if (shift != NO_PLACE) {
        pos = r + shift;
        const int page = __ldcg(a.block_table + (int64_t)i * a.table_stride + (pos >> a.b_shift));
        slot = ((int64_t)page << a.b_shift) + (pos & ((1 << a.b_shift) - 1));
    }
    a.slot_map[r] = slot;
    a.positions[r] = pos;
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(const PlanArgs a, const int rows_here) {
    __shared__ longlong2 s_warp[2 * PLAN_WARPS];
    __shared__ int32_t s_before[PLAN_THREADS], s_held[PLAN_THREADS], s_row0[PLAN_THREADS + 1], s_shift[PLAN_THREADS];
    __shared__ int s_taken;
    const int tid = threadIdx.x, b = 1 << a.b_shift;
    // pages that a sequence can hold: what a table's row has beyond them (up to its stride) is nobody's
    const int most = (int)(((int64_t)a.t_cap + b - 1) >> a.b_shift);
    pdl_wait();
    if (!rows_here) pdl_trigger();          // the rows' kernel, which waits for this one
    int n_free = __ldcg(a.n_free);
    // the first 1024 sequences' numbers at once, before anything is waited for (cold, every one of them is a microsecond)
    int32_t fresh0 = 0, gone0 = 0, len0 = 0;
    auto fetch = [&](int i, int32_t& fresh, int32_t& gone, int32_t& len) {
        fresh = gone = len = 0;
        if (i >= a.batch) return;
        if (a.release) gone = __ldcg(a.release + i);
        len = __ldcg(a.seq_lens + i);
        fresh = __ldcg(a.new_lens + i);
    };
    fetch(tid, fresh0, gone0, len0);
    n_free = n_free < 0 ? 0 : (n_free > a.n_pages ? a.n_pages : n_free);
    bool refused = false;

    // ---- pages of released sequences go back
    if (a.release) {
        for (int c = 0; c < a.batch; c += PLAN_THREADS) {
            int32_t fresh = fresh0, gone = gone0, len = len0;
            if (c) fetch(c + tid, fresh, gone, len);
            if (gone != 0) {
                gone = len <= 0 ? 0 : (int)(((int64_t)len + b - 1) >> a.b_shift);
                if (gone > most) { gone = most; refused = true; }
            }
            longlong2 all;
            s_before[tid] = saturated(scan(gone, 0, all, s_warp).x);
            __syncthreads();
            if (all.x > a.n_pages - n_free) { all.x = a.n_pages - n_free; refused = true; }      // more than were ever handed out
            const int n_seq = min(PLAN_THREADS, a.batch - c), n = (int)all.x;
            move_pages(s_before, n_seq, n, [&](int s, int p) { return __ldcg(a.block_table + (int64_t)(c + s) * a.table_stride + (p - s_before[s])); },
                       [&](int, int p, int page) { a.free_pages[n_free + p] = page; });
            n_free += n;
            __syncthreads();
        }
    }

    // ---- new tokens.  One scan serves rows and pages: the rows of a sequence lie within n_rows only if those of all before it do, so
    // among those that can be served the pages asked for before them are those of sequences that fit.
    int64_t rows_done = 0, pages_done = 0;       // rows and pages asked for so far, those that could not be had included
    int taken = 0;
    const bool one_chunk = a.batch <= PLAN_THREADS;
    for (int c = 0; c < a.batch; c += PLAN_THREADS) {
        const int i = c + tid, n_seq = min(PLAN_THREADS, a.batch - c);
        int32_t fresh = fresh0, gone = gone0, len = len0;
        if (c) fetch(i, fresh, gone, len);
        fresh = max(0, fresh);
        len = gone != 0 ? 0 : max(0, len);
        int held = 0, need = 0;
        bool fits = (int64_t)len + fresh <= a.t_cap;
        if (fits) {
            held = (int)(((int64_t)len + b - 1) >> a.b_shift);
            need = (int)(((int64_t)len + fresh + b - 1) >> a.b_shift) - held;
        }
        longlong2 all;
        if (tid == 0) s_taken = INT32_MAX;
        const longlong2 before = scan(fresh, need, all, s_warp);
        const int64_t row0 = rows_done + before.x, first = pages_done + before.y;
        fits = fits && row0 + fresh <= a.n_rows;
        const bool ok = fits && (need == 0 || first + need <= n_free);
        // Once a sequence that needs pages gets none, so do all later ones that need any: the pages taken are those asked for before the first such.
        if (!ok && need > 0) atomicMin(&s_taken, saturated(before.y));
        const int got = ok ? fresh : 0;
        s_before[tid] = saturated(before.y);
        s_held[tid] = held;
        s_row0[tid] = saturated(row0);
        s_shift[tid] = shift_of(len + got, got, saturated(row0));
        if (i < a.batch) {
            refused = refused || got != fresh;
            a.granted[i] = got;
            a.seq_lens_out[i] = len + got;
            a.row_start[i] = saturated(row0);
            if (i == a.batch - 1) a.row_start[a.batch] = s_row0[n_seq] = saturated(row0 + fresh);
        }
        __syncthreads();
        const int n = (int)(s_taken < all.y ? s_taken : all.y);
        move_pages(s_before, n_seq, n, [&](int, int p) { return __ldcg(a.free_pages + n_free - 1 - taken - p); },
                   [&](int s, int p, int page) { a.block_table[(int64_t)(c + s) * a.table_stride + s_held[s] + (p - s_before[s])] = page; });
        taken += n;
        rows_done += all.x;
        pages_done += all.y;
        __syncthreads();
    }
    if (tid == 0) *a.n_free_out = n_free - taken;
    if (refused && a.status) atomicOr(a.status, ETA_DEV_REFUSED);
    if (!rows_here) return;
    for (int r = tid; r < a.n_rows; r += PLAN_THREADS) {
        int i = 0;
        int32_t shift = NO_PLACE;
        if (one_chunk) {
            if (r < s_row0[a.batch]) {
                i = last_not_above(s_row0, a.batch, r);
                shift = s_shift[i];
            }
        } else if (r < __ldcg(a.row_start + a.batch)) {
            i = last_not_above_in_memory(a.row_start, a.batch, r);
            shift = shift_of(__ldcg(a.seq_lens_out + i), __ldcg(a.granted + i), __ldcg(a.row_start + i));
        }
        store_row(a, r, i, shift);
    }
}

// The rows of a large step, ROWS_PER_CTA to a CTA: which sequences they can belong to is one sweep over the row starts; what the rows need
// of those is put into shared memory where there is room, so that a row waits for its page's number only.
constexpr int ROWS_THREADS = 256, ROWS_PER_CTA = 1024, ROWS_SEQS = 1024;
__global__ void __launch_bounds__(ROWS_THREADS) plan_rows_kernel(const PlanArgs a) {
    __shared__ int s_first, s_last;
    __shared__ int32_t s_row0[ROWS_SEQS], s_shift[ROWS_SEQS];
    const int tid = threadIdx.x, r0 = blockIdx.x * ROWS_PER_CTA, r1 = min(a.n_rows, r0 + ROWS_PER_CTA);
    if (tid == 0) { s_first = 0; s_last = 0; }
    pdl_wait();
    __syncthreads();
    int first = 0, last = 0;
    for (int i = tid; i <= a.batch; i += ROWS_THREADS) {
        const int v = __ldcg(a.row_start + i);
        first += v <= r0;
        last += v <= r1 - 1;
    }
    first = __reduce_add_sync(0xffffffffu, first);
    last = __reduce_add_sync(0xffffffffu, last);
    if ((tid & 31) == 0) { atomicAdd(&s_first, first); atomicAdd(&s_last, last); }
    __syncthreads();
    const int lo = s_first - 1, n = s_last - lo;         // row_start[0] = 0: at least one is not above r0
    const bool near = n <= ROWS_SEQS;
    auto shift_at = [&](int i) {
        return i < a.batch ? shift_of(__ldcg(a.seq_lens_out + i), __ldcg(a.granted + i), __ldcg(a.row_start + i)) : NO_PLACE;
    };
    if (near) {
        for (int k = tid; k < n; k += ROWS_THREADS) {
            s_row0[k] = __ldcg(a.row_start + lo + k);
            s_shift[k] = shift_at(lo + k);
        }
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < ROWS_PER_CTA / ROWS_THREADS; ++u) {
        const int r = r0 + tid + u * ROWS_THREADS;
        if (r >= r1) break;
        const int k = near ? last_not_above(s_row0, n, r) : last_not_above_in_memory(a.row_start + lo, n, r);
        store_row(a, r, lo + k, near ? s_shift[k] : shift_at(lo + k));
    }
}

}  // namespace eta

extern "C" int eta_plan_pages(int32_t batch, int32_t block_size, int32_t t_cap, const int32_t* new_lens, const int32_t* release,
                              const int32_t* seq_lens, int32_t* seq_lens_out, int32_t* block_table, int32_t table_stride,
                              int32_t* free_pages, const int32_t* n_free, int32_t* n_free_out, int32_t n_pages, int32_t n_rows,
                              int64_t* slot_map, int32_t* positions, int32_t* row_start, int32_t* granted, uint32_t* status_dev,
                              void* stream) {
    using namespace eta;
    if (batch <= 0 || t_cap <= 0 || table_stride <= 0 || n_pages <= 0 || n_rows < 0) return ETA_ERR_INVALID_ARG;
    if (block_size != 32 && block_size != 64 && block_size != 128) return ETA_ERR_UNSUPPORTED;
    if ((int64_t)table_stride * block_size < t_cap) return ETA_ERR_INVALID_ARG;
    if (!new_lens || !seq_lens || !seq_lens_out || !block_table || !free_pages || !n_free || !n_free_out || !row_start || !granted)
        return ETA_ERR_INVALID_ARG;
    if (n_rows > 0 && (!slot_map || !positions)) return ETA_ERR_INVALID_ARG;
    if (batch > (1 << 30) || n_rows > (1 << 30) || n_pages > (1 << 30) || reinterpret_cast<uintptr_t>(slot_map) & 7) return ETA_ERR_UNSUPPORTED;
    PlanArgs a;
    a.batch = batch; a.b_shift = block_size == 32 ? 5 : (block_size == 64 ? 6 : 7);
    a.t_cap = t_cap; a.table_stride = table_stride; a.n_pages = n_pages; a.n_rows = n_rows;
    a.new_lens = new_lens; a.release = release; a.seq_lens = seq_lens; a.n_free = n_free;
    a.seq_lens_out = seq_lens_out; a.n_free_out = n_free_out; a.block_table = block_table; a.free_pages = free_pages;
    a.positions = positions; a.row_start = row_start; a.granted = granted; a.slot_map = slot_map; a.status = status_dev;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int rows_here = n_rows <= 4096;
    const int rc = launch_pdl("eta_plan_pages", plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, a, rows_here);
    if (rc != ETA_OK || rows_here) return rc;
    return launch_pdl("eta_plan_pages", plan_rows_kernel, dim3((unsigned)((n_rows + (int64_t)ROWS_PER_CTA - 1) / ROWS_PER_CTA)), dim3(ROWS_THREADS),
                      0, s, a);
}
