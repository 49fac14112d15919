// Block tables and slot maps of a paged cache from request lengths: what a serving loop does between two steps, on the GPU, so that
// the step can be captured and the host need not know the lengths.
//
//   released sequences:  their ceil(len / b) pages go on top of the free stack, sequence after sequence
//   new tokens:          need_i = ceil((len_i + new_i) / b) - ceil(len_i / b) pages come off its top, sequence after sequence
//   row r of sequence i: position p = len_i + (r - row_start_i), slot = table[i][p / b] * b + p % b
//
// Everything that depends on an order hangs on three prefix sums over the sequences (rows, pages back, pages needed): plan_kernel
// is one CTA that scans them 1024 sequences at a time, and moves the pages with a thread per page (found in the scan by
// bisection), so that a few long prompts do not leave it to a few threads.  The rows are its work too while they are few; beyond
// that a kernel over all rows follows.
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

// The sum of x over the threads before this one; `all`: over all of them.  Every thread of the CTA calls it; s_warp may be used again at once
// (its first half is read before the second barrier only, its second half is written after the next call's first).
__device__ __forceinline__ int64_t scan(int64_t x, int64_t& all, int64_t* s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t upto = x;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, upto, s);
        if (lane >= s) upto += o;
    }
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        int64_t w = s_warp[lane];
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t o = __shfl_up_sync(0xffffffffu, w, s);
            if (lane >= s) w += o;
        }
        s_warp[PLAN_WARPS + lane] = w;
    }
    __syncthreads();
    all = s_warp[2 * PLAN_WARPS - 1];
    return (warp ? s_warp[PLAN_WARPS + warp - 1] : 0) + upto - x;
}

// the last of n ascending numbers, the first of which is not above x, that is not above x
__device__ __forceinline__ int last_not_above(const int32_t* v, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Slot and position of row r, whose sequence is i (or none: i >= batch).
__device__ __forceinline__ void store_row(const PlanArgs& a, int r, int i) {
    int64_t slot = -1;
    int pos = 0;
    if (i < a.batch) {
        const int got = __ldcg(a.granted + i);
        if (got > 0) {
            pos = __ldcg(a.seq_lens_out + i) - got + (r - __ldcg(a.row_start + i));
            const int page = __ldcg(a.block_table + (int64_t)i * a.table_stride + (pos >> a.b_shift));
            slot = ((int64_t)page << a.b_shift) + (pos & ((1 << a.b_shift) - 1));
        }
    }
    a.slot_map[r] = slot;
    a.positions[r] = pos;
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(const PlanArgs a, const int rows_here) {
    __shared__ int64_t s_warp[2 * PLAN_WARPS];
    __shared__ int32_t s_before[PLAN_THREADS];
    const int tid = threadIdx.x, b = 1 << a.b_shift;
    pdl_wait();
    if (!rows_here) pdl_trigger();          // the rows' kernel, which waits for this one
    int n_free = __ldcg(a.n_free);
    n_free = n_free < 0 ? 0 : (n_free > a.n_pages ? a.n_pages : n_free);
    bool refused = false;

    // ---- pages of released sequences go back
    if (a.release) {
        for (int c = 0; c < a.batch; c += PLAN_THREADS) {
            const int i = c + tid;
            int gone = 0;
            if (i < a.batch && __ldcg(a.release + i) != 0) {
                const int len = __ldcg(a.seq_lens + i);
                gone = len <= 0 ? 0 : (int)(((int64_t)len + b - 1) >> a.b_shift);
                if (gone > a.table_stride) { gone = a.table_stride; refused = true; }
            }
            int64_t all;
            const int64_t before = scan(gone, all, s_warp);
            s_before[tid] = (int32_t)(before > INT32_MAX ? INT32_MAX : before);
            __syncthreads();
            if (all > a.n_pages - n_free) { all = a.n_pages - n_free; refused = true; }      // more than were ever handed out
            const int n_seq = min(PLAN_THREADS, a.batch - c);
            for (int p = tid; p < (int)all; p += PLAN_THREADS) {
                const int s = last_not_above(s_before, n_seq, p);
                a.free_pages[n_free + p] = __ldcg(a.block_table + (int64_t)(c + s) * a.table_stride + (p - s_before[s]));
            }
            n_free += (int)all;
            __syncthreads();
        }
    }

    // ---- new tokens
    int64_t rows_done = 0, pages_done = 0;       // rows and pages asked for so far, those that could not be had included
    int taken = 0;
    for (int c = 0; c < a.batch; c += PLAN_THREADS) {
        const int i = c + tid, n_seq = min(PLAN_THREADS, a.batch - c);
        int len = 0, fresh = 0, held = 0, need = 0;
        if (i < a.batch) {
            fresh = max(0, __ldcg(a.new_lens + i));
            len = a.release && __ldcg(a.release + i) != 0 ? 0 : max(0, __ldcg(a.seq_lens + i));
        }
        int64_t all_rows, all_need;
        const int64_t row0 = rows_done + scan(fresh, all_rows, s_warp);
        const bool fits = (int64_t)len + fresh <= a.t_cap && row0 + fresh <= a.n_rows;
        if (fits) {
            held = (int)(((int64_t)len + b - 1) >> a.b_shift);
            need = (int)(((int64_t)len + fresh + b - 1) >> a.b_shift) - held;
        }
        const int64_t first = pages_done + scan(need, all_need, s_warp);
        const bool ok = fits && (need == 0 || first + need <= n_free);
        if (i < a.batch) {
            const int got = ok ? fresh : 0;
            refused = refused || got != fresh;
            a.granted[i] = got;
            a.seq_lens_out[i] = len + got;
            a.row_start[i] = (int32_t)(row0 > INT32_MAX ? INT32_MAX : row0);
            if (i == a.batch - 1) a.row_start[a.batch] = (int32_t)(row0 + fresh > INT32_MAX ? INT32_MAX : row0 + fresh);
        }
        // Once a sequence that needs pages gets none, `first` is past the stack for all later ones: those that get pages come
        // first, and the pages asked for before them are the pages taken before them.
        int64_t taken_here;
        s_before[tid] = (int32_t)scan(ok ? need : 0, taken_here, s_warp);
        __syncthreads();
        for (int p = tid; p < (int)taken_here; p += PLAN_THREADS) {
            const int s = last_not_above(s_before, n_seq, p);
            const int l = __ldcg(a.seq_lens_out + c + s) - __ldcg(a.granted + c + s);
            const int at = (int)(((int64_t)l + b - 1) >> a.b_shift) + (p - s_before[s]);
            a.block_table[(int64_t)(c + s) * a.table_stride + at] = a.free_pages[n_free - 1 - taken - p];
        }
        taken += (int)taken_here;
        rows_done += all_rows;
        pages_done += all_need;
        __syncthreads();
    }
    if (tid == 0) *a.n_free_out = n_free - taken;
    if (refused && a.status) atomicOr(a.status, ETA_DEV_REFUSED);
    if (!rows_here) return;
    for (int r = tid; r < a.n_rows; r += PLAN_THREADS)
        store_row(a, r, r < __ldcg(a.row_start + a.batch) ? last_not_above(a.row_start, a.batch + 1, r) : a.batch);
}

// The rows of a large step, ROWS_PER_CTA to a CTA: which sequences they can belong to is one sweep over the row starts, then
// every row bisects among those.
constexpr int ROWS_THREADS = 256, ROWS_PER_CTA = 1024;
__global__ void __launch_bounds__(ROWS_THREADS) plan_rows_kernel(const PlanArgs a) {
    __shared__ int s_first, s_last;
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
    for (int r = r0 + tid; r < r1; r += ROWS_THREADS) store_row(a, r, lo + last_not_above(a.row_start + lo, n, r));
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
