// Block tables and slot maps of a paged key-value cache from request lengths, in one launch.
//
// Pages and slots of a request follow from exclusive prefix sums over the requests before it: pages given back, pages wanted, tokens added.
// One cluster does it all, so no second launch and no flag in memory is needed: every block reads and scans all requests for itself,
// nothing passes between blocks, and its share of the maps follows; cluster barriers keep what is updated in place from being written
// before every block has read it.  A few bytes per request and 8 per new token: bound by latency (loads, scan, cluster barriers, stores).
// Measured: 256 requests with a token each 7.8 us, 1024 requests of up to 512 new tokens 23 us, most of it the maps' 2 MB
// through 8 SMs.  (For steps of that size alone a second launch over all SMs, 2 to 3 us, could write the maps; not built.)
#include "nm_common.cuh"

namespace {

// What one request asks for.
struct PlanStep {
    int len, add;            // tokens it has, tokens it gets
    int held, wanted, back;  // pages it holds, pages it lacks, pages it returns
    int error;
};
struct PlanArgs {
    nm_kv_plan_desc d;
    NmDivisor by_page;
    uint32_t pages;   // page numbers below this one have slots of 31 bits
    int* status;
    int ctas, wide;   // wide: slots and positions are 16-byte aligned
};
__device__ __forceinline__ PlanStep plan_step(const PlanArgs& p, int i)
{
    const nm_kv_plan_desc& a = p.d;
    PlanStep s = {0, 0, 0, 0, 0, 0};
    if (i >= a.B) return s;
    const int len = a.lengths[i], add = a.new_tokens[i];
    const long long room = (long long)a.max_pages * a.page_size;   // fits 31 bits (checked by the entry point)
    s.len = len;
    if (len < 0 || len > room) {
        s.error = NM_ERR_INVALID_ARG;
        return s;
    }
    s.held = len ? p.by_page(len - 1) + 1 : 0;
    if (add < 0) {
        s.back = s.held;
        return s;
    }
    if ((long long)len + add > room) {
        s.error = NM_ERR_SHAPE;
        return s;
    }
    s.add = add;
    s.wanted = (len + add ? p.by_page(len + add - 1) + 1 : 0) - s.held;
    return s;
}

// Sums of the block's threads before this one (exclusive) and of all of them, three numbers at a time: within the warps, then the
// warps' sums within the first warp.
struct Sum3 {
    long long add, wanted, back;
};
__device__ __forceinline__ Sum3 warp_scan(Sum3 x, int lane)
{
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
    return x;
}
template <int THREADS> __device__ __forceinline__ Sum3 scan3(Sum3 v, Sum3* total, Sum3* s_warp)
{
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Sum3 x = warp_scan(v, lane);
    __syncthreads();   // the previous scan's sums have been read
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    if (warp == 0) {
        const Sum3 y = warp_scan(lane < WARPS ? s_warp[lane] : Sum3{0, 0, 0}, lane);
        __syncwarp();
        if (lane < WARPS) s_warp[lane] = y;
    }
    __syncthreads();
    const Sum3 before = warp ? s_warp[warp - 1] : Sum3{0, 0, 0};
    *total = s_warp[WARPS - 1];
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
// One tile, the usual case, is read and added up once.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) kv_plan_kernel(const PlanArgs p)
{
    const nm_kv_plan_desc& a = p.d;
    __shared__ Sum3 s_warp[THREADS / 32];
    __shared__ int s_start[THREADS], s_page[THREADS], s_back[THREADS], s_len[THREADS], s_held[THREADS];
    __shared__ int s_error;
    const int tid = threadIdx.x, rank = blockIdx.x, gtid = rank * THREADS + tid, gthreads = p.ctas * THREADS;
    const int tiles = (a.B + THREADS - 1) / THREADS;
    if (tid == 0) s_error = 0;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    __syncthreads();
    const int count = *a.free_count;

    // what the whole step asks for
    PlanStep step = {0, 0, 0, 0, 0, 0};
    Sum3 mine = {0, 0, 0}, all;
    for (int t = 0; t < tiles; ++t) {
        step = plan_step(p, t * THREADS + tid);
        mine.add += step.add;
        mine.wanted += step.wanted;
        mine.back += step.back;
        if (step.error == NM_ERR_INVALID_ARG) atomicOr(&s_error, 4);
        if (step.error == NM_ERR_SHAPE) atomicOr(&s_error, 2);
    }
    Sum3 before = scan3<THREADS>(mine, &all, s_warp);
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
            atomicExch(p.status, bad & 4 ? (int)NM_ERR_INVALID_ARG : bad & 2 ? (int)NM_ERR_SHAPE : (int)NM_ERR_WORKSPACE);
        }
        return;
    }
    const int top = (int)(count + all.back) - 1;   // of the stack, once all released pages are on it

    if (all.back > 0) {
        int done = 0;
        for (int t = 0; t < tiles; ++t) {
            Sum3 sum = all;
            if (tiles > 1) {
                step = plan_step(p, t * THREADS + tid);
                before = scan3<THREADS>(Sum3{step.add, step.wanted, step.back}, &sum, s_warp);
            }
            s_back[tid] = (int)before.back;
            __syncthreads();
            for (int x = gtid; x < (int)sum.back; x += gthreads) {
                const int r = owner_of(s_back, THREADS, x);
                a.free_pages[count + done + x] = a.block_tables[(int64_t)(t * THREADS + r) * a.ld_tables + x - s_back[r]];
            }
            done += (int)sum.back;
        }
    }
    if (tiles > 1) nm_cluster_sync();

    int token0 = 0, page0 = 0;   // tokens and taken pages of the tiles before
    for (int t = 0; t < tiles; ++t) {
        const int i = t * THREADS + tid;
        Sum3 sum = all;
        if (tiles > 1) {
            step = plan_step(p, i);
            before = scan3<THREADS>(Sum3{step.add, step.wanted, step.back}, &sum, s_warp);
        }
        const bool over = i < a.B && a.new_tokens[i] < 0;
        s_start[tid] = (int)before.add;
        s_page[tid] = (int)before.wanted;
        s_len[tid] = step.len;
        s_held[tid] = step.held;
        __syncthreads();
        nm_cluster_sync();   // every CTA has read this tile's lengths; released pages are on the stack
        if (rank == 0 && i < a.B) {
            a.lengths_out[i] = over ? 0 : step.len + step.add;
            a.token_start[i] = token0 + (int)before.add;
        }
        for (int x = gtid; x < (int)sum.wanted; x += gthreads) {
            const int r = owner_of(s_page, THREADS, x);
            a.block_tables[(int64_t)(t * THREADS + r) * a.ld_tables + s_held[r] + x - s_page[r]] = a.free_pages[top - page0 - x];
        }
        // Four tokens a thread, one search for them; what belongs to the tile is [token0, token0 + sum.add) of the arrays.
        const int n = (int)sum.add, lead = token0 & 3;   // fours begin at multiples of four of the arrays
        for (int x0 = gtid * 4 - lead; x0 < n; x0 += gthreads * 4) {
            const int first = x0 < 0 ? 0 : x0;
            int r = owner_of(s_start, THREADS, first), page = -1, entry_of = -1;
            int slot[4] = {-1, -1, -1, -1}, position[4] = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int x = x0 + k;
                if (x < 0 || x >= n) continue;
                while (r + 1 < THREADS && s_start[r + 1] <= x) {   // the next request that has tokens
                    ++r;
                    entry_of = -1;
                }
                const int pos = s_len[r] + x - s_start[r], entry = p.by_page(pos);
                if (entry != entry_of) {
                    // a page that the request lacked comes from the stack: its table entry may not be written yet
                    page = entry < s_held[r] ? a.block_tables[(int64_t)(t * THREADS + r) * a.ld_tables + entry]
                                             : a.free_pages[top - page0 - (s_page[r] + entry - s_held[r])];
                    entry_of = entry;
                }
                if ((uint32_t)page < p.pages) slot[k] = page * a.page_size + (pos - entry * a.page_size);
                else atomicExch(p.status, (int)NM_ERR_INVALID_ARG);
                position[k] = pos;
            }
            const int at = token0 + x0;
            if (p.wide && x0 >= 0 && x0 + 4 <= n) {
                *reinterpret_cast<int4*>(a.slots + at) = make_int4(slot[0], slot[1], slot[2], slot[3]);
                *reinterpret_cast<int4*>(a.positions + at) = make_int4(position[0], position[1], position[2], position[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (x0 + k >= 0 && x0 + k < n) {
                        a.slots[at + k] = slot[k];
                        a.positions[at + k] = position[k];
                    }
            }
        }
        token0 += (int)sum.add;
        page0 += (int)sum.wanted;
        __syncthreads();   // the tile's arrays have been read
    }
    if (tiles == 0) nm_cluster_sync();
    for (int x = token0 + gtid; x < a.max_tokens; x += gthreads) {
        a.slots[x] = -1;
        a.positions[x] = 0;
    }
    if (gtid == 0) {
        a.token_start[a.B] = token0;
        *a.free_count_out = top + 1 - page0;
    }
}

template <int THREADS> nm_status launch(nm_ctx* ctx, const PlanArgs& p, cudaStream_t st)
{
    NmLaunchScope scope(ctx, NM_KERNEL_KV_PLAN, 16.0 * p.d.B + 8.0 * p.d.max_tokens, st);
    NmLaunchConfig lc(ctx, dim3(p.ctas), THREADS, 0, st, p.ctas);
    return cudaLaunchKernelEx(&lc.cfg, kv_plan_kernel<THREADS>, p) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

}  // namespace

nm_status nm_launch_kv_plan(nm_ctx* ctx, const nm_kv_plan_desc* d, cudaStream_t st)
{
    PlanArgs p;
    p.d = *d;
    p.by_page = NmDivisor::of(d->page_size);
    p.pages = (uint32_t)((1ll << 31) / d->page_size);
    p.status = ctx->d_status;
    p.wide = nm_aligned16(d->slots) && nm_aligned16(d->positions);
    // A step of few requests and tokens is a chain of latencies: one small block (B 256: 10.8 us with 1024 threads and three scans).
    // Otherwise the largest portable cluster.
    const bool small = d->max_tokens <= 4 * 1024;
    p.ctas = small ? 1 : 8;
    return small && d->B <= 256 ? launch<256>(ctx, p, st) : launch<1024>(ctx, p, st);
}
