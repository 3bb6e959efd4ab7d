// Pages of the paged cache, handed out on the device: request lengths are device data (how many documents survive pruning is
// decided there), so block tables and slot maps are built there too, and no length visits the host between two steps.
//
// cf_pages_resize is a handful of prefix sums over the requests and as many writes as pages and slots change.  The free pages
// are a stack.  Releases go first, last request and last column first, then the growing requests take pages in order:
// growing and shrinking back leaves the stack as it was, and who gets which page does not depend on timing.
#include <algorithm>
#include <climits>

#include "cf_kv4.cuh"

namespace cf {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kAtOnce = 4;                        // released columns whose loads a lane has under way
constexpr int kFillSlots = 2048;                  // slots of a block of fill_kernel

__device__ __forceinline__ int cluster_rank() {
    int r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ int cluster_size() {
    int n;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}
// What the blocks of the cluster have written before is visible to all behind it.
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Inclusive prefix sums of a and b over the block; totals in ta and tb.  `sums` holds 66 ints.
__device__ __forceinline__ void scan2(int& a, int& b, int& ta, int& tb, int* sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) a += x, b += y;
    }
    __syncthreads();                                        // the previous round's readers are done
    if (lane == 31) sums[warp] = a, sums[33 + warp] = b;
    __syncthreads();
    if (warp == 0) {
        int x = lane < n_warps ? sums[lane] : 0, y = lane < n_warps ? sums[33 + lane] : 0;
        const int x0 = x, y0 = y;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int p = __shfl_up_sync(0xffffffffu, x, o), q = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) x += p, y += q;
        }
        sums[lane] = x - x0, sums[33 + lane] = y - y0;
        if (lane == 31) sums[32] = x, sums[65] = y;
    }
    __syncthreads();
    a += sums[warp], b += sums[33 + warp];
    ta = sums[32], tb = sums[65];
}

// What a request asks for, and whether its length and the slot map allow it.
struct Wish {
    int before, after, have, need;
    bool fits;
};

__device__ __forceinline__ Wish wish_of(const PagesView& pv, Divisor page_rows, int max_new, int before, int rows, int extra) {
    Wish w;
    const int most = pv.table_cols * pv.page_rows;
    const long long asked = rows < 0 ? 0 : (long long)rows + extra;
    w.before = max(0, min(before, most));
    w.fits = asked >= 0 && asked <= most && (max_new < 0 || asked - w.before <= max_new);
    w.after = w.fits ? (int)asked : w.before;
    w.have = page_rows.quotient(w.before + pv.page_rows - 1);
    w.need = page_rows.quotient(w.after + pv.page_rows - 1);
    return w;
}

// The slot of row `row` of a request that had `have` pages, the k-th of its new ones lying k below `top` on the stack.
__device__ __forceinline__ long long slot_of(const PagesView& pv, Divisor page_rows, const int* table, int row, int have, int top) {
    const int c = page_rows.quotient(row);
    const int page = c < have ? table[c] : pv.free_pages[top - (c - have)];
    return (long long)page * pv.page_rows + (row - c * pv.page_rows);
}

// One cluster: who gets what.  Each of its blocks takes all prefix sums; pages that are released, and columns and slots that are
// filled here (`fill`), are shared out among the blocks, request by request to their warps.  Without `fill` a request's former
// length and stack place are left in the first entry of every kFillSlots of its slots, for fill_kernel.  `target` may be the
// lengths that the pages hold: they are written behind a barrier that every reader has passed.
__global__ void __launch_bounds__(kPlanThreads)
resize_kernel(PagesView pv, Divisor page_rows, Divisor per_request, const int* target, int extra, int max_new, long long* slots, int fill) {
    chain_next();
    chain_wait();
    __shared__ int s_sums[66];
    __shared__ int s_before[kPlanThreads], s_after[kPlanThreads], s_at[kPlanThreads];
    __shared__ int s_given;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
    const int rank = cluster_rank(), blocks = cluster_size(), first_warp = warp * blocks + rank, all_warps = n_warps * blocks;
    const int n = pv.n_requests, limit = slots ? max_new : -1;
    const bool one = n <= (int)blockDim.x;                  // one round of the block: its sums are taken once
    const int height = max(0, min(pv.n_pages, *pv.free_count));
    if (tid == 0) s_given = 0;
    Wish w = {};
    int back, sum, all_back, all_sum;                       // pages released and asked for up to this request, and in the round
    auto round = [&](int b) {
        w = Wish{};
        if (b < n) w = wish_of(pv, page_rows, limit, pv.rows[b], target[b], extra);
        back = max(0, w.have - w.need), sum = max(0, w.need - w.have);
        scan2(back, sum, all_back, all_sum, s_sums);
    };
    int released = 0;
    bool wrong = false;
    for (int b0 = 0; b0 < n; b0 += blockDim.x) {
        round(b0 + tid);
        released += all_back;
    }
    const int top = min(pv.n_pages, height + released);     // the stack's height once they are back
    if (released > 0) {
        int earlier = 0;
        for (int b0 = 0; b0 < n; b0 += blockDim.x) {
            if (!one) round(b0 + tid);
            s_before[tid] = w.have, s_after[tid] = min(w.have, w.need);
            s_at[tid] = height + released - (earlier + back);   // place of the last column's page
            __syncthreads();
            for (int j = first_warp; j < min((int)blockDim.x, n - b0); j += all_warps) {
                int* table = pv.table + (size_t)(b0 + j) * pv.table_cols;
                const int last = s_before[j] - 1, place = s_at[j];
                for (int c0 = s_after[j] + lane; c0 <= last; c0 += 32 * kAtOnce) {
                    int page[kAtOnce];
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) page[i] = c0 + 32 * i <= last ? table[c0 + 32 * i] : 0;
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) {
                        const int c = c0 + 32 * i, at = place + last - c;
                        if (c > last) break;
                        wrong |= (unsigned)page[i] >= (unsigned)pv.n_pages || at >= pv.n_pages;
                        if (at < pv.n_pages) pv.free_pages[at] = page[i];
                        table[c] = -1;
                    }
                }
            }
            earlier += all_back;
            __syncthreads();
        }
    }
    // growing requests, in order
    int asked = 0;
    bool beyond = false, short_of = false;
    for (int b0 = 0; b0 < n; b0 += blockDim.x) {
        const int b = b0 + tid;
        if (!one) round(b);
        cluster_barrier();                                  // lengths read, released pages on the stack
        const int mine = max(0, w.need - w.have);
        const bool served = w.fits && (mine == 0 || asked + sum <= top);
        beyond |= b < n && !w.fits;
        short_of |= b < n && w.fits && !served;
        // those that are served come before all that are not: what they take together is the largest of their sums
        if (served && mine > 0) atomicMax(&s_given, asked + sum);
        const int place = top - 1 - (asked + sum - mine);
        s_before[tid] = w.before, s_after[tid] = served ? w.after : w.before, s_at[tid] = place;
        if (b < n && rank == 0) pv.rows[b] = s_after[tid];
        asked += all_sum;
        __syncthreads();
        const int chunk = min((int)blockDim.x, n - b0);
        if (fill) {
            for (int j = first_warp; j < chunk; j += all_warps) {           // columns: a warp to a request
                const int have = page_rows.quotient(s_before[j] + pv.page_rows - 1), need = page_rows.quotient(s_after[j] + pv.page_rows - 1);
                for (int c = have + lane; c < need; c += 32) pv.table[(size_t)(b0 + j) * pv.table_cols + c] = pv.free_pages[s_at[j] - (c - have)];
            }
            // slots: a thread to each
            for (int x = rank * blockDim.x + tid; x < chunk * max_new; x += blocks * blockDim.x) {
                const int j = per_request.quotient(x), row = s_before[j] + per_request.remainder(x);
                slots[(size_t)b0 * max_new + x] = row >= s_after[j] ? -1 : slot_of(pv, page_rows, pv.table + (size_t)(b0 + j) * pv.table_cols, row,
                                                                                   page_rows.quotient(s_before[j] + pv.page_rows - 1), s_at[j]);
            }
        } else if (b < n && rank == 0) {
            for (long long i = 0; i < max_new; i += kFillSlots) slots[(size_t)b * max_new + i] = (long long)place * (1LL << 32) + w.before;
        }
        __syncthreads();
    }
    if (wrong) atomicCAS(pv.status, 0, CF_ERR_INVALID_ARG);
    beyond = __syncthreads_or(beyond), short_of = __syncthreads_or(short_of);
    if (tid == 0 && rank == 0) {
        if (beyond || short_of) atomicCAS(pv.status, 0, beyond ? CF_ERR_RANGE : CF_ERR_WORKSPACE);
        *pv.free_count = top - s_given;
    }
}

// A block per kFillSlots slots of a request, which fills them and its part of the columns.
__global__ void __launch_bounds__(kFillThreads)
fill_kernel(PagesView pv, Divisor page_rows, int max_new, long long* slots) {
    chain_next();
    chain_wait();
    const int b = blockIdx.x, slot0 = blockIdx.y * kFillSlots;
    const long long left = slots[(size_t)b * max_new + slot0];
    const int after = pv.rows[b];
    __syncthreads();                                        // everyone has it before it is overwritten
    const int before = (int)(left & 0xffffffffLL), top = (int)(left >> 32);
    const int have = page_rows.quotient(before + pv.page_rows - 1), need = page_rows.quotient(after + pv.page_rows - 1);
    int* table = pv.table + (size_t)b * pv.table_cols;
    for (int c = have + blockIdx.y * kFillThreads + threadIdx.x; c < need; c += gridDim.y * kFillThreads) table[c] = pv.free_pages[top - (c - have)];
    const int end = min(max_new, slot0 + kFillSlots);
#pragma unroll 4
    for (int i = slot0 + threadIdx.x; i < end; i += kFillThreads) {
        const long long row = (long long)before + i;
        slots[(size_t)b * max_new + i] = row >= after ? -1 : slot_of(pv, page_rows, table, (int)row, have, top);
    }
}

__global__ void __launch_bounds__(256)
pages_init_kernel(PagesView pv) {
    chain_next();
    chain_wait();
    const long long first = blockIdx.x * 256LL + threadIdx.x, step = gridDim.x * 256LL;
    for (long long i = first; i < (long long)pv.n_requests * pv.table_cols; i += step) pv.table[i] = -1;
    for (long long i = first; i < pv.n_requests; i += step) pv.rows[i] = 0;
    for (long long i = first; i < pv.n_pages; i += step) pv.free_pages[i] = pv.n_pages - 1 - (int)i;
    if (first == 0) {
        *pv.free_count = pv.n_pages;
        *pv.status = 0;
    }
}

// The blocks that plan write columns and slots themselves where there are few: a step's new rows.
bool fill_in_place(int n_requests, int max_new) { return max_new <= 64 && (long long)n_requests * max_new <= 16384; }

}  // namespace

int check_pages(const cf_pages* p) {
    if (!p || p->n_requests <= 0 || p->n_requests > (1 << 20) || p->page_rows < 16 || p->page_rows % 16 != 0 || p->n_pages <= 0 ||
        p->table_cols <= 0)
        return CF_ERR_INVALID_ARG;
    if ((long long)p->table_cols * p->page_rows > INT_MAX - 2LL * p->page_rows - 256 || (long long)p->n_requests * p->table_cols + p->n_pages > INT_MAX)
        return CF_ERR_INVALID_ARG;                // the stack's height, while pages come back, is counted in 32 bits
    if (!p->table || !p->rows || !p->free_pages || !p->free_count || !p->status) return CF_ERR_INVALID_ARG;
    return CF_OK;
}

PagesView make_pages_view(const cf_pages* p) {
    return {p->n_requests, p->page_rows, p->n_pages, p->table_cols, p->table, p->rows, p->free_pages, p->free_count, p->status};
}

}  // namespace cf

using namespace cf;

extern "C" {

int cf_pages_init(const cf_pages* pages, void* stream) {
    const int rc = check_pages(pages);
    if (rc != CF_OK) return rc;
    return launch_chained(pages_init_kernel, dim3(128), 256, 0, static_cast<cudaStream_t>(stream), make_pages_view(pages));
}

int cf_pages_resize(const cf_pages* pages, const int32_t* rows, int32_t extra_rows, int32_t max_new, int64_t* slots, void* stream) {
    const int rc = check_pages(pages);
    if (rc != CF_OK) return rc;
    if (!rows || max_new < 0 || max_new > 65535 * kFillSlots || (max_new > 0) != (slots != nullptr)) return CF_ERR_INVALID_ARG;
    const PagesView pv = make_pages_view(pages);
    const Divisor page_rows(pages->page_rows);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool fill = fill_in_place(pages->n_requests, max_new);
    const int threads = std::min(kPlanThreads, std::max(128, (pages->n_requests + 31) / 32 * 32));
    long long* map = reinterpret_cast<long long*>(slots);
    // eight blocks share what there is to write (one block / eight, us: a step of 16 requests 2.3 / 2.3, of 256 5.6 / 3.3, of 1000
    // 9.0 / 5.1; 1021 requests of which 90 end and 100 arrive 21.7 / 9.0)
    const unsigned cluster = pages->n_requests >= 8 ? 8 : 1;
    const int err = launch_chained_clusters(resize_kernel, dim3(cluster), threads, 0, cluster, s, pv, page_rows, Divisor(std::max(1, max_new)), rows,
                                            extra_rows, max_new, map, fill ? 1 : 0);
    if (err != CF_OK || fill) return err;
    return launch_chained(fill_kernel, dim3((unsigned)pages->n_requests, (unsigned)((max_new + kFillSlots - 1) / kFillSlots)), kFillThreads, 0, s, pv,
                          page_rows, max_new, map);
}

int cf_pages_status(const cf_pages* pages, void* stream) {
    const int rc = check_pages(pages);
    if (rc != CF_OK) return rc;
    int32_t word = 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(&word, pages->status, sizeof(word), cudaMemcpyDeviceToHost, s) != cudaSuccess) return CF_ERR_CUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return CF_ERR_CUDA;
    return word;
}

}  // extern "C"
