// k_plan.hip -- pages, slots and per-token lists of a batch from its requests' lengths.
//
// With have_b = ceil(ctx_b / 16), pages_b = ceil((ctx_b + new_b) / 16) - have_b of the valid rows
// and their inclusive prefix sums cp, ct over pages and tokens, row b is admitted when cp_b <= n_free
// and ct_b <= max_tokens: both sums only grow, so the admitted rows are the valid ones before the
// first that does not fit, and no row's answer waits for another's.
// One launch: every block repeats the prefix sums of all rows (at most 1024, four a thread) in LDS and
// then writes its share of the tokens, the new page-table entries and the per-row outputs, each found by
// a binary search in the sums.  A token on a page that its row held before reads the page table, one on
// a new page the free list, so no block waits for what another writes.
// Bound by the launch and one chain of reads: 64 rows of one token 4.5 us, 256 rows with 261 thousand tokens (3.3 MB
// written) 6.3 us of a captured graph; the smallest launch takes 4.0.
#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {

constexpr int PL_THREADS = 256;
constexpr int PL_ROWS = PLAN_MAXB / PL_THREADS;  // rows a thread sums

// The last row r < B with sum[r] <= i (sum[0] = 0, ascending, i < sum[B]): the row that holds element i.
__device__ __forceinline__ int row_of(const int* sum, int B, int i) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(PL_THREADS) void batch_plan_kernel(PlanArgs a) {
    __shared__ int tok0[PLAN_MAXB + 1], pg0[PLAN_MAXB + 1], ctx_s[PLAN_MAXB];
    __shared__ long long wt[PL_THREADS / 64], wp[PL_THREADS / 64];
    __shared__ int stop_s;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int n_free = max(a.n_free[0], 0);
    const long long cap = 16ll * a.maxp;

    // rows PL_ROWS t .. + 3: their tokens and pages, the thread's own prefix, then the block's
    int ctx[PL_ROWS], nw[PL_ROWS], np[PL_ROWS];
    bool valid[PL_ROWS];
    long long st = 0, sp = 0;
#pragma unroll
    for (int k = 0; k < PL_ROWS; ++k) {
        const int b = PL_ROWS * t + k;
        const int c = b < a.B ? a.ctx[b] : -1, n = b < a.B ? a.n_new[b] : 0;
        valid[k] = c >= 0 && n >= 0 && (long long)c + n <= cap;
        ctx[k] = c;
        nw[k] = valid[k] ? n : 0;
        np[k] = valid[k] ? (int)(((long long)c + n + 15) / 16 - ((long long)c + 15) / 16) : 0;
        st += nw[k];
        sp += np[k];
    }
    long long it = st, ip = sp;  // inclusive over the wave's threads
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long ut = __shfl_up(it, o, 64), up = __shfl_up(ip, o, 64);
        if (lane >= o) { it += ut; ip += up; }
    }
    if (lane == 63) { wt[wave] = it; wp[wave] = ip; }
    if (t == 0) stop_s = a.B;
    __syncthreads();
    long long ct = it - st, cp = ip - sp;  // exclusive over the block's threads
    for (int w = 0; w < wave; ++w) { ct += wt[w]; cp += wp[w]; }
    // the first valid row that does not fit: every valid row behind it does not either
    int stop = a.B;
    {
        long long c = ct, p = cp;
#pragma unroll
        for (int k = PL_ROWS - 1; k >= 0; --k) { c += nw[k]; p += np[k]; }
#pragma unroll
        for (int k = PL_ROWS - 1; k >= 0; --k) {
            if (valid[k] && (p > n_free || c > a.max_tokens)) stop = min(stop, PL_ROWS * t + k);
            c -= nw[k];
            p -= np[k];
        }
    }
    if (stop < a.B) atomicMin(&stop_s, stop);
    __syncthreads();
    stop = stop_s;
#pragma unroll
    for (int k = 0; k < PL_ROWS; ++k) {
        const int b = PL_ROWS * t + k;
        if (b <= stop) {  // the sums before it passed no limit
            tok0[b] = (int)ct;
            pg0[b] = (int)cp;
        }
        if (b < a.B) {
            ctx_s[b] = ctx[k];
            if (blockIdx.x == 0) {
                const bool ok = valid[k] && b < stop;
                a.admitted[b] = ok;
                a.lens[b] = max(ctx[k], 0) + (ok ? nw[k] : 0);
            }
        }
        ct += nw[k];
        cp += np[k];
        if (b == PLAN_MAXB - 1 && stop == PLAN_MAXB) {
            tok0[PLAN_MAXB] = (int)ct;
            pg0[PLAN_MAXB] = (int)cp;
        }
    }
    __syncthreads();
    const int total = tok0[stop], pages = pg0[stop];
    for (int b = stop + 1 + t; b <= a.B; b += PL_THREADS) {
        tok0[b] = total;
        pg0[b] = pages;
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int b = t; b <= a.B; b += PL_THREADS) a.cu_new[b] = tok0[b];
        if (t == 0) a.n_left[0] = n_free - pages;
    }
    const int stride = gridDim.x * PL_THREADS, first = blockIdx.x * PL_THREADS + t;
    for (int i = first; i < pages; i += stride) {
        const int r = row_of(pg0, a.B, i);
        a.page_table[(size_t)r * a.maxp + (ctx_s[r] + 15) / 16 + i - pg0[r]] = a.free_pages[n_free - 1 - i];
    }
    for (int i = first; i < a.max_tokens; i += stride) {
        int pos = -1, row = -1, slot = -1;
        if (i < total) {
            row = row_of(tok0, a.B, i);
            pos = ctx_s[row] + i - tok0[row];
            const int have = (ctx_s[row] + 15) / 16, pg = pos / 16;
            const int page = pg < have ? a.page_table[(size_t)row * a.maxp + pg] : a.free_pages[n_free - 1 - (pg0[row] + pg - have)];
            slot = (uint32_t)page < 1u << 27 ? page * 16 + pos % 16 : -1;  // (any other id's slot would be another page's)
        }
        a.positions[i] = pos;
        a.rows[i] = row;
        a.slots[i] = slot;
    }
}

hipError_t launch_batch_plan(const PlanArgs& a, hipStream_t s) {
    const int blocks = min(max((a.max_tokens + PL_THREADS - 1) / PL_THREADS, 1), 1024);
    hipLaunchKernelGGL(batch_plan_kernel, dim3(blocks), dim3(PL_THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace mg
