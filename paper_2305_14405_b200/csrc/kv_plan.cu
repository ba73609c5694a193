// Block tables and slot maps of a paged key-value cache from request lengths, in one launch.
#include "nm_common.cuh"

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_TILE = PLAN_THREADS;   // one request of a tile per thread

// What one request asks for.
struct PlanStep {
    int len, add;            // tokens it has, tokens it gets
    int held, wanted, back;  // pages it holds, pages it lacks, pages it returns
    int error;
};
__device__ __forceinline__ PlanStep plan_step(const nm_kv_plan_desc& a, int i)
{
    PlanStep s = {0, 0, 0, 0, 0, 0};
    if (i >= a.B) return s;
    const int len = a.lengths[i], add = a.new_tokens[i];
    const long long room = (long long)a.max_pages * a.page_size;   // fits 31 bits (checked by the entry point)
    s.len = len;
    if (len < 0 || len > room) {
        s.error = NM_ERR_INVALID_ARG;
        return s;
    }
    s.held = (int)(((long long)len + a.page_size - 1) / a.page_size);
    if (add < 0) {
        s.back = s.held;
        return s;
    }
    if ((long long)len + add > room) {
        s.error = NM_ERR_SHAPE;
        return s;
    }
    s.add = add;
    s.wanted = (int)(((long long)len + add + a.page_size - 1) / a.page_size) - s.held;
    return s;
}

// Sums of the block's threads before this one (exclusive) and of all of them, three numbers at a time.
struct Sum3 {
    long long add, wanted, back;
};
__device__ __forceinline__ Sum3 scan3(Sum3 v, Sum3* total, Sum3* s_warp)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sum3 x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, x.add, o), w = __shfl_up_sync(0xffffffffu, x.wanted, o),
                        b = __shfl_up_sync(0xffffffffu, x.back, o);
        if (lane >= o) {
            x.add += a;
            x.wanted += w;
            x.back += b;
        }
    }
    __syncthreads();   // the previous scan's sums have been read
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    Sum3 before = {0, 0, 0}, all = {0, 0, 0};
    for (int w = 0; w < PLAN_THREADS / 32; ++w) {
        const Sum3 y = s_warp[w];
        if (w == warp) before = all;
        all.add += y.add;
        all.wanted += y.wanted;
        all.back += y.back;
    }
    *total = all;
    return Sum3{before.add + x.add - v.add, before.wanted + x.wanted - v.wanted, before.back + x.back - v.back};
}

// Last index i of the first n with start[i] <= x (start[0] <= x).
__device__ __forceinline__ int owner_of(const int* start, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// One cluster.  Every CTA reads all requests and adds them up for itself, in tiles of one request per thread, so that nothing
// has to be passed between CTAs; the tokens, pages and released pages of a tile are then spread over the cluster's threads, each
// finding its request by a search among the tile's starts.  All that a step reads and writes in place is separated by barriers
// of the cluster: released pages are on the stack before the first is taken, a tile's lengths are read by all before one is written.
__global__ void __launch_bounds__(PLAN_THREADS) kv_plan_kernel(const nm_kv_plan_desc a, int* __restrict__ status, int ctas)
{
    __shared__ Sum3 s_warp[PLAN_THREADS / 32];
    __shared__ int s_start[PLAN_TILE], s_page[PLAN_TILE], s_len[PLAN_TILE], s_held[PLAN_TILE];
    __shared__ int s_error;
    const int tid = threadIdx.x, rank = blockIdx.x, gtid = rank * PLAN_THREADS + tid, gthreads = ctas * PLAN_THREADS;
    const int tiles = (a.B + PLAN_TILE - 1) / PLAN_TILE;
    if (tid == 0) s_error = 0;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    __syncthreads();
    const int count = *a.free_count;

    // what the whole step asks for
    Sum3 mine = {0, 0, 0}, all;
    for (int t = 0; t < tiles; ++t) {
        const PlanStep s = plan_step(a, t * PLAN_TILE + tid);
        mine.add += s.add;
        mine.wanted += s.wanted;
        mine.back += s.back;
        if (s.error == NM_ERR_INVALID_ARG) atomicOr(&s_error, 4);
        if (s.error == NM_ERR_SHAPE) atomicOr(&s_error, 2);
    }
    (void)scan3(mine, &all, s_warp);
    int bad = s_error;
    if (count < 0 || count > a.free_capacity || count + all.back > a.free_capacity) bad |= 4;
    if (all.add > a.max_tokens) bad |= 2;
    if (all.wanted > count + all.back) bad |= 1;
    if (bad) {   // the same decision in every CTA: nothing is changed
        nm_cluster_sync();
        for (int i = gtid; i < a.B; i += gthreads) a.lengths_out[i] = a.lengths[i];
        for (int i = gtid; i <= a.B; i += gthreads) a.token_start[i] = 0;
        for (int i = gtid; i < a.max_tokens; i += gthreads) {
            a.slots[i] = -1;
            a.positions[i] = 0;
        }
        if (gtid == 0) {
            *a.free_count_out = count;
            atomicExch(status, bad & 4 ? (int)NM_ERR_INVALID_ARG : bad & 2 ? (int)NM_ERR_SHAPE : (int)NM_ERR_WORKSPACE);
        }
        return;
    }
    const int top = (int)(count + all.back) - 1;   // of the stack, once all released pages are on it

    if (all.back > 0) {
        int done = 0;
        for (int t = 0; t < tiles; ++t) {
            const PlanStep s = plan_step(a, t * PLAN_TILE + tid);
            Sum3 sum;
            const Sum3 before = scan3(Sum3{0, 0, s.back}, &sum, s_warp);
            s_start[tid] = (int)before.back;
            __syncthreads();
            for (int x = gtid; x < (int)sum.back; x += gthreads) {
                const int r = owner_of(s_start, PLAN_TILE, x);
                a.free_pages[count + done + x] = a.block_tables[(int64_t)(t * PLAN_TILE + r) * a.ld_tables + x - s_start[r]];
            }
            done += (int)sum.back;
        }
    }
    nm_cluster_sync();

    int token0 = 0, page0 = 0;   // tokens and taken pages of the tiles before
    for (int t = 0; t < tiles; ++t) {
        const int i = t * PLAN_TILE + tid;
        const PlanStep s = plan_step(a, i);
        Sum3 sum;
        const Sum3 before = scan3(Sum3{s.add, s.wanted, 0}, &sum, s_warp);
        s_start[tid] = (int)before.add;
        s_page[tid] = (int)before.wanted;
        s_len[tid] = s.len;
        s_held[tid] = s.held;
        __syncthreads();
        nm_cluster_sync();   // every CTA has read this tile's lengths
        if (rank == 0 && i < a.B) {
            a.lengths_out[i] = s.back > 0 || a.new_tokens[i] < 0 ? 0 : s.len + s.add;
            a.token_start[i] = token0 + (int)before.add;
        }
        for (int x = gtid; x < (int)sum.wanted; x += gthreads) {
            const int r = owner_of(s_page, PLAN_TILE, x);
            a.block_tables[(int64_t)(t * PLAN_TILE + r) * a.ld_tables + s_held[r] + x - s_page[r]] = a.free_pages[top - page0 - x];
        }
        for (int x = gtid; x < (int)sum.add; x += gthreads) {
            const int r = owner_of(s_start, PLAN_TILE, x);
            const int pos = s_len[r] + x - s_start[r], entry = pos / a.page_size;
            // a page that the request lacked comes from the stack: its table entry may not be written yet
            const int page = entry < s_held[r] ? a.block_tables[(int64_t)(t * PLAN_TILE + r) * a.ld_tables + entry]
                                               : a.free_pages[top - page0 - (s_page[r] + entry - s_held[r])];
            a.slots[token0 + x] = page * a.page_size + pos % a.page_size;
            a.positions[token0 + x] = pos;
        }
        token0 += (int)sum.add;
        page0 += (int)sum.wanted;
        __syncthreads();   // the tile's arrays have been read
    }
    for (int x = token0 + gtid; x < a.max_tokens; x += gthreads) {
        a.slots[x] = -1;
        a.positions[x] = 0;
    }
    if (gtid == 0) {
        a.token_start[a.B] = token0;
        *a.free_count_out = top + 1 - page0;
    }
}

}  // namespace

nm_status nm_launch_kv_plan(nm_ctx* ctx, const nm_kv_plan_desc* d, cudaStream_t st)
{
    // one CTA where it writes every token and request in one go, otherwise the largest portable cluster
    const int ctas = d->B <= PLAN_THREADS && d->max_tokens <= PLAN_THREADS ? 1 : 8;
    NmLaunchScope scope(ctx, NM_KERNEL_KV_PLAN, 16.0 * d->B + 8.0 * d->max_tokens, st);
    NmLaunchConfig lc(ctx, dim3(ctas), PLAN_THREADS, 0, st, ctas);
    const nm_kv_plan_desc a = *d;
    return cudaLaunchKernelEx(&lc.cfg, kv_plan_kernel, a, ctx->d_status, ctas) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}
