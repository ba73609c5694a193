// Attention of one new token per request over a paged key-value cache with PWL softmax.
//
// A PWL exponential is not multiplicative, so e_j = PWL_exp(s_j - m) needs the maximum m of the whole row before the first
// value is weighted: a running maximum that rescales earlier sums would compute another function.  Keys and values are still
// read once each: the scores (4 bytes per token and head, against 2 d elements of K and V per token and key head) are kept.
//   1. scores:   a block per request, key head and span of tokens multiplies K; scores and the span's maximum to the workspace
//   2. values:   the same blocks, now with the row's maximum, weight V; partial sums to the workspace (or, with one span, the result)
//   3. join:     the spans' sums of each head added in their order, times PWL_recip of the row sum
// Everything that leaves the row of a span is fp32.
#include "nm_common.cuh"

namespace {

constexpr int PAGED_THREADS = 128, PAGED_WARPS = PAGED_THREADS / 32;

struct PagedArgs {
    nm_attn_paged_desc d;
    const NmTable *exp_tab, *recip_tab;
    int* status;
    int group, blocks_per_head;   // query heads of a key head; blocks of HB of them
    int span, spans;              // tokens per block, blocks per row
    int64_t row;                  // scores of one head in the workspace
    float *scores, *maxima, *sums, *outs;   // [B][heads][row], [B][heads][spans], [B][heads][spans], [B][heads][spans][d]
};

__device__ __forceinline__ float paged_table(const NmTable* t, float x)
{
    const float2 kb = t->kb[nm_pwl_index(x, t->inv_h, t->off, (float)(t->n - 1))];
    return __fmaf_rn(kb.x, x, kb.y);
}

// The length of request b, or -1 where it is outside what the call was made for (recorded; nothing is written then).
__device__ __forceinline__ int paged_length(const PagedArgs& a, int b)
{
    const int n = a.d.lengths[b];
    if (n < 0 || n > a.d.max_len) {
        if (threadIdx.x == 0) atomicExch(a.status, (int)NM_ERR_SHAPE);
        return -1;
    }
    return n;
}

// Element offset of token j's page and place, or -1 for a page that the cache does not have (recorded).
__device__ __forceinline__ int64_t paged_token(const PagedArgs& a, const int32_t* table, int j)
{
    const int entry = j / a.d.page_size, page = table[entry];
    if (page < 0 || page >= a.d.num_pages) {
        atomicExch(a.status, (int)NM_ERR_INVALID_ARG);
        return -1;
    }
    return (int64_t)page * a.d.stride_page + (int64_t)(j - entry * a.d.page_size) * a.d.stride_token;
}

template <typename T> struct Vec16 {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ void get(float* f) const
    {
        const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = NmType<T>::to_f(e[i]);
    }
};

struct PagedBlock {
    int b, kv, h0, nh, span;   // request, key head, first query head, query heads, span of tokens
};
template <int HB> __device__ __forceinline__ PagedBlock paged_block(const PagedArgs& a)
{
    PagedBlock p;
    int64_t x = blockIdx.x;
    p.span = (int)(x % a.spans);
    x /= a.spans;
    const int hb = (int)(x % a.blocks_per_head);
    x /= a.blocks_per_head;
    p.kv = (int)(x % a.d.kv_heads);
    p.b = (int)(x / a.d.kv_heads);
    p.h0 = p.kv * a.group + hb * HB;
    p.nh = min(HB, a.group - hb * HB);
    return p;
}

// LPK lanes hold a key, VPL vectors of 16 bytes each (lanes behind the head's channels hold none), so a warp works on 32/LPK
// keys at a time against HB query heads in registers.
template <typename T, int LPK, int VPL, int HB>
__global__ void __launch_bounds__(PAGED_THREADS) paged_scores_kernel(const PagedArgs a)
{
    constexpr int N = Vec16<T>::N, KPW = 32 / LPK;
    __shared__ float s_max[PAGED_WARPS][HB];
    const PagedBlock p = paged_block<HB>(a);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane & (LPK - 1), sub = lane / LPK;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, p.b), first = p.span * a.span;
    if (first >= len) return;
    const int last = min(len, first + a.span);
    float q[HB][VPL][N], m[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        m[h] = -INFINITY;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const int c = (v * LPK + part) * N;
            Vec16<T> x;
            x.raw = make_uint4(0, 0, 0, 0);
            if (h < p.nh && c < a.d.d)
                x.raw = *reinterpret_cast<const uint4*>((const T*)a.d.Q + (int64_t)p.b * a.d.ld_q + (int64_t)(p.h0 + h) * a.d.d + c);
            x.get(q[h][v]);
        }
    }
    const int32_t* table = a.d.block_tables + (int64_t)p.b * a.d.ld_tables;
    const T* K = (const T*)a.d.k_cache + (int64_t)p.kv * a.d.stride_head;
    for (int j0 = first + warp * KPW; j0 < last; j0 += PAGED_WARPS * KPW) {
        const int j = j0 + sub;
        const int64_t at = j < last ? paged_token(a, table, j) : -1;
        float dot[HB];
#pragma unroll
        for (int h = 0; h < HB; ++h) dot[h] = 0.f;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const int c = (v * LPK + part) * N;
            Vec16<T> x;
            x.raw = make_uint4(0, 0, 0, 0);
            if (at >= 0 && c < a.d.d) x.raw = *reinterpret_cast<const uint4*>(K + at + c);
            float k[N];
            x.get(k);
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int i = 0; i < N; ++i) dot[h] = __fmaf_rn(q[h][v][i], k[i], dot[h]);
        }
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int o = LPK / 2; o > 0; o >>= 1) dot[h] += __shfl_xor_sync(0xffffffffu, dot[h], o);
        if (j < last) {
#pragma unroll
            for (int h = 0; h < HB; ++h) {
                const float s = dot[h] * a.d.scale;
                m[h] = fmaxf(m[h], s);
                if (part == 0 && h < p.nh) a.scores[((int64_t)p.b * a.d.heads + p.h0 + h) * a.row + j] = s;
            }
        }
    }
#pragma unroll
    for (int h = 0; h < HB; ++h) {
#pragma unroll
        for (int o = 16; o >= LPK; o >>= 1) m[h] = fmaxf(m[h], __shfl_xor_sync(0xffffffffu, m[h], o));
        if (lane == 0) s_max[warp][h] = m[h];
    }
    __syncthreads();
    if ((int)threadIdx.x < p.nh) {
        float x = s_max[0][threadIdx.x];
        for (int w = 1; w < PAGED_WARPS; ++w) x = fmaxf(x, s_max[w][threadIdx.x]);
        a.maxima[((int64_t)p.b * a.d.heads + p.h0 + threadIdx.x) * a.spans + p.span] = x;
    }
}

template <typename T, int LPK, int VPL, int HB>
__global__ void __launch_bounds__(PAGED_THREADS) paged_values_kernel(const PagedArgs a)
{
    constexpr int N = Vec16<T>::N, KPW = 32 / LPK;
    __shared__ float s_m[HB], s_sum[PAGED_WARPS][HB], s_out[PAGED_WARPS][HB][LPK * VPL * N];
    const PagedBlock p = paged_block<HB>(a);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane & (LPK - 1), sub = lane / LPK;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, p.b), first = p.span * a.span;
    if (first >= len) return;
    const int last = min(len, first + a.span), used = (len + a.span - 1) / a.span;
    for (int h = warp; h < HB; h += PAGED_WARPS) {
        float m = -INFINITY;
        if (h < p.nh)
            for (int i = lane; i < used; i += 32) m = fmaxf(m, a.maxima[((int64_t)p.b * a.d.heads + p.h0 + h) * a.spans + i]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) s_m[h] = m;
    }
    __syncthreads();
    float acc[HB][VPL][N], sum[HB], m[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        sum[h] = 0.f;
        m[h] = s_m[h];
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) acc[h][v][i] = 0.f;
    }
    const int32_t* table = a.d.block_tables + (int64_t)p.b * a.d.ld_tables;
    const T* V = (const T*)a.d.v_cache + (int64_t)p.kv * a.d.stride_head;
    for (int j0 = first + warp * KPW; j0 < last; j0 += PAGED_WARPS * KPW) {
        const int j = j0 + sub;
        if (j >= last) continue;
        const int64_t at = paged_token(a, table, j);
        float e[HB];
#pragma unroll
        for (int h = 0; h < HB; ++h) {
            e[h] = h < p.nh ? paged_table(a.exp_tab, a.scores[((int64_t)p.b * a.d.heads + p.h0 + h) * a.row + j] - m[h]) : 0.f;
            sum[h] += e[h];
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const int c = (v * LPK + part) * N;
            Vec16<T> x;
            x.raw = make_uint4(0, 0, 0, 0);
            if (at >= 0 && c < a.d.d) x.raw = *reinterpret_cast<const uint4*>(V + at + c);
            float f[N];
            x.get(f);
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int i = 0; i < N; ++i) acc[h][v][i] = __fmaf_rn(e[h], f[i], acc[h][v][i]);
        }
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < HB; ++h) {
#pragma unroll
        for (int o = 16; o >= LPK; o >>= 1) {
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], o);
#pragma unroll
            for (int v = 0; v < VPL; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) acc[h][v][i] += __shfl_xor_sync(0xffffffffu, acc[h][v][i], o);
        }
        if (sub == 0) {
#pragma unroll
            for (int v = 0; v < VPL; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) s_out[warp][h][(v * LPK + part) * N + i] = acc[h][v][i];
        }
        if (lane == 0) s_sum[warp][h] = sum[h];
    }
    __syncthreads();
    for (int x = threadIdx.x; x < p.nh * a.d.d; x += PAGED_THREADS) {
        const int h = x / a.d.d, c = x - h * a.d.d;
        float o = s_out[0][h][c], s = s_sum[0][h];
        for (int w = 1; w < PAGED_WARPS; ++w) {
            o += s_out[w][h][c];
            s += s_sum[w][h];
        }
        const int64_t row = ((int64_t)p.b * a.d.heads + p.h0 + h) * a.spans + p.span;
        a.outs[row * a.d.d + c] = o;
        if (c == 0) a.sums[row] = s;
    }
}

// A block per request and head.
template <typename T>
__global__ void __launch_bounds__(PAGED_THREADS) paged_join_kernel(const PagedArgs a)
{
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.d.heads), h = (int)(bh - (int64_t)b * a.d.heads);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, b);
    if (len < 0) return;
    const int used = (len + a.span - 1) / a.span;
    float s = 0.f;
    for (int i = 0; i < used; ++i) s += a.sums[bh * a.spans + i];
    const float r = paged_table(a.recip_tab, s);
    for (int c = threadIdx.x; c < a.d.d; c += PAGED_THREADS) {
        float o = 0.f;
        for (int i = 0; i < used; ++i) o += a.outs[(bh * a.spans + i) * a.d.d + c];
        ((T*)a.d.out)[(int64_t)b * a.d.ld_out + (int64_t)h * a.d.d + c] = NmType<T>::from_f(used ? o * r : 0.f);
    }
}

int heads_per_block(int group) { return group >= 8 ? 8 : group >= 4 ? 4 : group >= 2 ? 2 : 1; }

struct PagedLayout {
    int hb, blocks_per_head, span, spans;
    int64_t row;
    size_t scores, maxima, sums, outs, total;
};
PagedLayout layout_of(const nm_attn_paged_desc* d)
{
    PagedLayout l;
    const int group = d->heads / d->kv_heads;
    l.hb = heads_per_block(group);
    l.blocks_per_head = (group + l.hb - 1) / l.hb;
    // spans of whole 128 tokens, as many as make eight blocks per SM of a 148-SM device
    const int64_t rows = (int64_t)d->B * d->kv_heads * l.blocks_per_head, tokens = (rows * d->max_len + 148 * 8 - 1) / (148 * 8);
    l.span = (int)(((tokens < 1 ? 1 : tokens > d->max_len ? d->max_len : tokens) + 127) / 128 * 128);
    l.spans = d->max_len > 0 ? (int)(((int64_t)d->max_len + l.span - 1) / l.span) : 1;
    l.row = ((int64_t)d->max_len + 31) / 32 * 32;
    const size_t bh = (size_t)d->B * d->heads;
    size_t o = 0;
    auto take = [&o](size_t bytes) { const size_t at = o; o += (bytes + 255) / 256 * 256; return at; };
    l.scores = take(bh * l.row * 4);
    l.maxima = take(bh * l.spans * 4);
    l.sums = take(bh * l.spans * 4);
    l.outs = take(bh * l.spans * d->d * 4);
    l.total = o;
    return l;
}

template <typename T, int LPK, int VPL, int HB>
nm_status launch(nm_ctx* ctx, const PagedArgs& a, int64_t blocks, cudaStream_t st)
{
    const double bytes = (double)a.d.B * a.d.max_len * a.d.kv_heads * a.d.d * sizeof(T);
    {
        NmLaunchScope scope(ctx, NM_KERNEL_ATTENTION_PAGED, bytes, st);
        NmLaunchConfig lc(ctx, dim3((unsigned)blocks), PAGED_THREADS, 0, st);
        if (cudaLaunchKernelEx(&lc.cfg, paged_scores_kernel<T, LPK, VPL, HB>, a) != cudaSuccess) return NM_ERR_CUDA;
    }
    {
        NmLaunchScope scope(ctx, NM_KERNEL_ATTENTION_PAGED, bytes, st);
        NmLaunchConfig lc(ctx, dim3((unsigned)blocks), PAGED_THREADS, 0, st);
        if (cudaLaunchKernelEx(&lc.cfg, paged_values_kernel<T, LPK, VPL, HB>, a) != cudaSuccess) return NM_ERR_CUDA;
    }
    NmLaunchScope scope(ctx, NM_KERNEL_ATTENTION_PAGED, 0.0, st);
    NmLaunchConfig lc(ctx, dim3((unsigned)(a.d.B * (int64_t)a.d.heads)), PAGED_THREADS, 0, st);
    return cudaLaunchKernelEx(&lc.cfg, paged_join_kernel<T>, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

template <typename T>
nm_status dispatch(nm_ctx* ctx, const PagedArgs& a, int hb, int64_t blocks, cudaStream_t st)
{
    const int vecs = a.d.d * (int)sizeof(T) / 16;
#define NM_PAGED_HB(LPK, VPL)                                                \
    do {                                                                     \
        if (hb == 8) return launch<T, LPK, VPL, 8>(ctx, a, blocks, st);      \
        if (hb == 4) return launch<T, LPK, VPL, 4>(ctx, a, blocks, st);      \
        if (hb == 2) return launch<T, LPK, VPL, 2>(ctx, a, blocks, st);      \
        return launch<T, LPK, VPL, 1>(ctx, a, blocks, st);                   \
    } while (0)
    if (vecs <= 8) NM_PAGED_HB(8, 1);
    if (vecs <= 16) NM_PAGED_HB(16, 1);
    if (vecs <= 32) NM_PAGED_HB(32, 1);
    if constexpr (sizeof(T) == 4) NM_PAGED_HB(32, 2);
#undef NM_PAGED_HB
    return NM_ERR_UNSUPPORTED;
}

}  // namespace

size_t nm_attention_paged_bytes(const nm_attn_paged_desc* d) { return layout_of(d).total; }

nm_status nm_launch_attention_paged(nm_ctx* ctx, const nm_attn_paged_desc* d, void* workspace, cudaStream_t st)
{
    const PagedLayout l = layout_of(d);
    PagedArgs a;
    a.d = *d;
    a.exp_tab = ctx->d_tables + d->exp_slot;
    a.recip_tab = ctx->d_tables + d->recip_slot;
    a.status = ctx->d_status;
    a.group = d->heads / d->kv_heads;
    a.blocks_per_head = l.blocks_per_head;
    a.span = l.span;
    a.spans = l.spans;
    a.row = l.row;
    a.scores = (float*)((uint8_t*)workspace + l.scores);
    a.maxima = (float*)((uint8_t*)workspace + l.maxima);
    a.sums = (float*)((uint8_t*)workspace + l.sums);
    a.outs = (float*)((uint8_t*)workspace + l.outs);
    const int64_t blocks = (int64_t)d->B * d->kv_heads * l.blocks_per_head * l.spans;
    if (blocks > INT32_MAX || (int64_t)d->B * d->heads > INT32_MAX) return NM_ERR_SHAPE;
    switch (d->dtype) {
    case NM_F32: return dispatch<float>(ctx, a, l.hb, blocks, st);
    case NM_BF16: return dispatch<__nv_bfloat16>(ctx, a, l.hb, blocks, st);
    case NM_F16: return dispatch<__half>(ctx, a, l.hb, blocks, st);
    default: return NM_ERR_UNSUPPORTED;
    }
}
