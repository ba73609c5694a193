// Attention of one new token per request over a paged key-value cache with PWL softmax.  Bound by the bytes of K and V.
//
// A PWL exponential is not multiplicative, so e_j = PWL_exp(s_j - m) needs the maximum m of the whole row before the first value is
// weighted: a running maximum that rescales earlier sums would compute another function.  Keys and values are still read once
// each, because the scores are kept (4 bytes per token and query head, against 2 d elements of K and V per token and key head):
//   fused   a cluster of blocks per request and key head, scores in shared memory, maxima and sums exchanged within the cluster
//   split   rows longer than a cluster holds: one launch for the scores (to the workspace), one for the values, one that joins
// A unit of work is a request, a key head and up to HEADS of its query heads; its tokens are split over blocks, a block's over its
// warps in tiles.  Two cores do a tile:
//   PagedMma   16-bit types, d a multiple of 32: m16n8k16 products, fragments loaded from the cache straight into registers
//   PagedFma   fp32 and other d: FMAs, a few lanes per token
// Partial sums are fp32 and are added in the order of warps and blocks: results do not depend on timing.
#include "nm_common.cuh"

namespace {

constexpr int PAGED_WARPS = 8, PAGED_THREADS = PAGED_WARPS * 32;

struct PagedArgs {
    nm_attn_paged_desc d;
    const NmTable *exp_tab, *recip_tab;
    int* status;
    int group, blocks_per_head;   // query heads of a key head; units that they make
    int span, spans;              // split: tokens of a block, blocks of a row; fused: tokens that a block's shared memory holds
    int64_t row;                  // split: scores of one head in the workspace
    float *scores, *maxima, *sums, *outs;   // split: [B][heads][row], [B][heads][spans], [B][heads][spans], [B][heads][spans][d]
};

__device__ __forceinline__ float paged_table(const NmTable* t, float x)
{
    const float2 kb = t->kb[nm_pwl_index(x, t->inv_h, t->off, (float)(t->n - 1))];
    return __fmaf_rn(kb.x, x, kb.y);
}

// The exponential's table in shared memory.
struct PagedExp {
    const float2* kb;
    float inv_h, off, nm1;
    __device__ __forceinline__ float operator()(float x) const
    {
        const float2 v = kb[nm_pwl_index(x, inv_h, off, nm1)];
        return __fmaf_rn(v.x, x, v.y);
    }
};

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

// Element offsets of the block's tokens in K and V (without the head); -1 for a page that the cache does not have (recorded).
__device__ __forceinline__ void paged_offsets(const PagedArgs& a, int b, int first, int count, int64_t* off)
{
    const int32_t* table = a.d.block_tables + (int64_t)b * a.d.ld_tables;
    for (int i = threadIdx.x; i < count; i += PAGED_THREADS) {
        const int j = first + i, entry = j / a.d.page_size, page = table[entry];
        if (page < 0 || page >= a.d.num_pages) {
            atomicExch(a.status, (int)NM_ERR_INVALID_ARG);
            off[i] = -1;
        } else {
            off[i] = (int64_t)page * a.d.stride_page + (int64_t)(j - entry * a.d.page_size) * a.d.stride_token;
        }
    }
}

// ---------------------------------------------------------------- tensor-core tiles

__device__ __forceinline__ void paged_mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void paged_mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// (a, b) as a pair of 16-bit numbers and what they leave of a and b
__device__ __forceinline__ uint32_t paged_term(float& a, float& b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    a -= __low2float(h);
    b -= __high2float(h);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t paged_term(float& a, float& b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    a -= __low2float(h);
    b -= __high2float(h);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Tiles of 16 tokens, NT tiles of 8 query heads.  Lane (g, t) = (lane / 4, lane % 4).
//   scores  S^T = K Q^T: lane (g, t) loads 16 bytes of tokens g and g + 8 in every 32 channels, which four of its neighbours make 64
//           contiguous bytes.  Which channel is which k of a product is free as long as Q has the same order.
//   values  O^T = V^T P^T: lane (g, t) loads 8 channels of tokens 2t, 2t + 1, 2t + 8, 2t + 9 in every 64 (4 in a last 32), so rows
//           are read 128 bytes at a time; a byte permutation pairs two tokens' channels.  Probabilities are two 16-bit terms.
template <typename T, int D_, int NT> struct PagedMma {
    using Elem = T;
    static constexpr int D = D_, HEADS = NT * 8, TILE = 16, WIDE = D / 64, NARROW = (D % 64) / 32;
    static_assert(D % 32 == 0, "whole 32-channel pieces");

    // put(h, i, s) takes the score of head h and token i; max_of(h) of the warp's scores is left in m for lane 0's readers
    template <typename Put>
    static __device__ __forceinline__ void scores(const PagedArgs& a, const T* Q, int nh, const T* K, const int64_t* off, int count, float* warp_max,
                                                  Put put)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
        uint4 q[NT][D / 32];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                q[n][c] = n * 8 + g < nh ? *reinterpret_cast<const uint4*>(Q + (n * 8 + g) * D + c * 32 + t * 8) : make_uint4(0, 0, 0, 0);
        float m[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) m[n][0] = m[n][1] = -INFINITY;
        for (int i0 = warp * TILE; i0 < count; i0 += PAGED_WARPS * TILE) {
            const int i = i0 + g;
            const int64_t at0 = i < count ? off[i] : -1, at1 = i + 8 < count ? off[i + 8] : -1;
            uint4 k0[D / 32], k1[D / 32];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                k0[c] = at0 >= 0 ? __ldg(reinterpret_cast<const uint4*>(K + at0 + c * 32 + t * 8)) : make_uint4(0, 0, 0, 0);
                k1[c] = at1 >= 0 ? __ldg(reinterpret_cast<const uint4*>(K + at1 + c * 32 + t * 8)) : make_uint4(0, 0, 0, 0);
            }
            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    paged_mma(s[n], k0[c].x, k1[c].x, k0[c].y, k1[c].y, q[n][c].x, q[n][c].y, T());
                    paged_mma(s[n], k0[c].z, k1[c].z, k0[c].w, k1[c].w, q[n][c].z, q[n][c].w, T());
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = s[n][r] * a.d.scale;
                    const int j = i + (r >> 1) * 8;
                    if (j < count) {
                        m[n][r & 1] = fmaxf(m[n][r & 1], v);
                        put(n * 8 + 2 * t + (r & 1), j, v);
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) m[n][r] = fmaxf(m[n][r], __shfl_xor_sync(0xffffffffu, m[n][r], o));
                if (g == 0) warp_max[n * 8 + 2 * t + r] = m[n][r];
            }
    }

    uint4 w0[WIDE ? WIDE : 1][4];   // values of tokens 2t, 2t + 1, 2t + 8, 2t + 9
    uint2 w1[4];
    __device__ __forceinline__ void load(const T* V, const int64_t* off, int i0, int count)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = i0 + 2 * t + (r & 1) + (r >> 1) * 8;
            const int64_t at = i < count ? off[i] : -1;
#pragma unroll
            for (int c = 0; c < WIDE; ++c)
                w0[c][r] = at >= 0 ? __ldg(reinterpret_cast<const uint4*>(V + at + c * 64 + g * 8)) : make_uint4(0, 0, 0, 0);
            if (NARROW) w1[r] = at >= 0 ? __ldg(reinterpret_cast<const uint2*>(V + at + WIDE * 64 + g * 4)) : make_uint2(0, 0);
        }
    }
    // get(h, i) gives the scores of head h and tokens i, i + 1; `first` is called once the first tile is on its way and gives the maxima
    template <typename Max, typename Get>
    __device__ __forceinline__ void values(const PagedArgs& a, int nh, const T* V, const int64_t* off, int count, PagedExp exp, float* warp_sum,
                                           float* warp_out, Max first, Get get)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
        float acc[NT][D / 16][4], sum[NT], m[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            sum[n] = 0.f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) acc[n][c][0] = acc[n][c][1] = acc[n][c][2] = acc[n][c][3] = 0.f;
        }
        int i0 = warp * TILE;
        if (i0 < count) load(V, off, i0, count);
        const float* maxima = first();
#pragma unroll
        for (int n = 0; n < NT; ++n) m[n] = maxima[n * 8 + g];
        while (i0 < count) {
            uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int i = i0 + 2 * t + r * 8;
                    float x = 0.f, y = 0.f;
                    if (n * 8 + g < nh && i < count) {
                        const float2 s = get(n * 8 + g, i);   // a row's storage has whole tiles
                        x = exp(s.x - m[n]);
                        y = i + 1 < count ? exp(s.y - m[n]) : 0.f;
                    }
                    sum[n] += x + y;
                    hi[n][r] = paged_term(x, y, T());
                    lo[n][r] = paged_term(x, y, T());
                }
            auto pair = [&](int c, uint32_t x0, uint32_t x1, uint32_t x8, uint32_t x9) {   // two channels of four tokens
                const uint32_t f0 = __byte_perm(x0, x1, 0x5410), f1 = __byte_perm(x0, x1, 0x7632), f2 = __byte_perm(x8, x9, 0x5410),
                               f3 = __byte_perm(x8, x9, 0x7632);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    paged_mma(acc[n][c], f0, f1, f2, f3, hi[n][0], hi[n][1], T());
                    paged_mma(acc[n][c], f0, f1, f2, f3, lo[n][0], lo[n][1], T());
                }
            };
#pragma unroll
            for (int c = 0; c < WIDE; ++c) {
                pair(c * 4 + 0, w0[c][0].x, w0[c][1].x, w0[c][2].x, w0[c][3].x);
                pair(c * 4 + 1, w0[c][0].y, w0[c][1].y, w0[c][2].y, w0[c][3].y);
                pair(c * 4 + 2, w0[c][0].z, w0[c][1].z, w0[c][2].z, w0[c][3].z);
                pair(c * 4 + 3, w0[c][0].w, w0[c][1].w, w0[c][2].w, w0[c][3].w);
            }
            if constexpr (NARROW != 0) {
                pair(WIDE * 4 + 0, w1[0].x, w1[1].x, w1[2].x, w1[3].x);
                pair(WIDE * 4 + 1, w1[0].y, w1[1].y, w1[2].y, w1[3].y);
            }
            i0 += PAGED_WARPS * TILE;
            if (i0 < count) load(V, off, i0, count);
        }
        __syncthreads();   // scores and offsets have been read: warp_out may lie over them
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
            sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
            if (t == 0) warp_sum[n * 8 + g] = sum[n];
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int ch = (c < WIDE * 4 ? (c >> 2) * 64 + g * 8 + (c & 3) * 2 : WIDE * 64 + g * 4 + (c - WIDE * 4) * 2) + (r >> 1);
                    warp_out[(n * 8 + 2 * t + (r & 1)) * D + ch] = acc[n][c][r];
                }
        }
    }
};

// ---------------------------------------------------------------- FMA tiles

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

// LPK lanes hold a token, VPL vectors of 16 bytes each (lanes behind the head's channels hold none): 32/LPK tokens at a time
// against HB query heads in registers.
template <typename T, int LPK, int VPL, int HB> struct PagedFma {
    using Elem = T;
    static constexpr int N = Vec16<T>::N, TILE = 32 / LPK, HEADS = HB, D = LPK * VPL * N;   // D: room for the channels

    template <typename Put>
    static __device__ __forceinline__ void scores(const PagedArgs& a, const T* Q, int nh, const T* K, const int64_t* off, int count, float* warp_max,
                                                  Put put)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane & (LPK - 1), sub = lane / LPK;
        float q[HB][VPL][N], m[HB];
#pragma unroll
        for (int h = 0; h < HB; ++h) {
            m[h] = -INFINITY;
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const int c = (v * LPK + part) * N;
                Vec16<T> x;
                x.raw = h < nh && c < a.d.d ? *reinterpret_cast<const uint4*>(Q + h * a.d.d + c) : make_uint4(0, 0, 0, 0);
                x.get(q[h][v]);
            }
        }
        for (int i0 = warp * TILE; i0 < count; i0 += PAGED_WARPS * TILE) {
            const int i = i0 + sub;
            const int64_t at = i < count ? off[i] : -1;
            float dot[HB];
#pragma unroll
            for (int h = 0; h < HB; ++h) dot[h] = 0.f;
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const int c = (v * LPK + part) * N;
                Vec16<T> x;
                x.raw = at >= 0 && c < a.d.d ? __ldg(reinterpret_cast<const uint4*>(K + at + c)) : make_uint4(0, 0, 0, 0);
                float k[N];
                x.get(k);
#pragma unroll
                for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int e = 0; e < N; ++e) dot[h] = __fmaf_rn(q[h][v][e], k[e], dot[h]);
            }
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int o = LPK / 2; o > 0; o >>= 1) dot[h] += __shfl_xor_sync(0xffffffffu, dot[h], o);
            if (i < count) {
#pragma unroll
                for (int h = 0; h < HB; ++h) {
                    const float s = dot[h] * a.d.scale;
                    m[h] = fmaxf(m[h], s);
                    if (part == 0 && h < nh) put(h, i, s);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < HB; ++h) {
#pragma unroll
            for (int o = 16; o >= LPK; o >>= 1) m[h] = fmaxf(m[h], __shfl_xor_sync(0xffffffffu, m[h], o));
            if (lane == 0) warp_max[h] = m[h];
        }
    }

    template <typename Max, typename Get>
    __device__ __forceinline__ void values(const PagedArgs& a, int nh, const T* V, const int64_t* off, int count, PagedExp exp, float* warp_sum,
                                           float* warp_out, Max first, Get get)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane & (LPK - 1), sub = lane / LPK;
        float acc[HB][VPL][N], sum[HB], m[HB];
        const float* maxima = first();
#pragma unroll
        for (int h = 0; h < HB; ++h) {
            sum[h] = 0.f;
            m[h] = maxima[h];
#pragma unroll
            for (int v = 0; v < VPL; ++v)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[h][v][e] = 0.f;
        }
        for (int i = warp * TILE + sub; i < count; i += PAGED_WARPS * TILE) {
            const int64_t at = off[i];
            Vec16<T> x[VPL];
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const int c = (v * LPK + part) * N;
                x[v].raw = at >= 0 && c < a.d.d ? __ldg(reinterpret_cast<const uint4*>(V + at + c)) : make_uint4(0, 0, 0, 0);
            }
            float e[HB];
#pragma unroll
            for (int h = 0; h < HB; ++h) {
                float s = 0.f;
                if (h < nh) {
                    const float2 two = get(h, i & ~1);
                    s = exp((i & 1 ? two.y : two.x) - m[h]);
                }
                e[h] = s;
                sum[h] += s;
            }
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                float f[N];
                x[v].get(f);
#pragma unroll
                for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int k = 0; k < N; ++k) acc[h][v][k] = __fmaf_rn(e[h], f[k], acc[h][v][k]);
            }
        }
        __syncthreads();   // scores and offsets have been read: warp_out may lie over them
#pragma unroll
        for (int h = 0; h < HB; ++h) {
#pragma unroll
            for (int o = 16; o >= LPK; o >>= 1) {
                sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], o);
#pragma unroll
                for (int v = 0; v < VPL; ++v)
#pragma unroll
                    for (int k = 0; k < N; ++k) acc[h][v][k] += __shfl_xor_sync(0xffffffffu, acc[h][v][k], o);
            }
            if (sub == 0) {
#pragma unroll
                for (int v = 0; v < VPL; ++v)
#pragma unroll
                    for (int k = 0; k < N; ++k) warp_out[h * D + (v * LPK + part) * N + k] = acc[h][v][k];
            }
            if (lane == 0) warp_sum[h] = sum[h];
        }
    }
};

// ---------------------------------------------------------------- kernels

struct PagedUnit {
    int b, kv, h0, nh;   // request, key head, first query head, query heads
};
template <class Core> __device__ __forceinline__ PagedUnit paged_unit(const PagedArgs& a, int64_t x)
{
    PagedUnit u;
    const int hb = (int)(x % a.blocks_per_head);
    x /= a.blocks_per_head;
    u.kv = (int)(x % a.d.kv_heads);
    u.b = (int)(x / a.d.kv_heads);
    u.h0 = u.kv * a.group + hb * Core::HEADS;
    u.nh = min(Core::HEADS, a.group - hb * Core::HEADS);
    return u;
}
template <class Core> __host__ __device__ constexpr size_t paged_out_bytes() { return (size_t)PAGED_WARPS * Core::HEADS * Core::D * 4; }
// scores of a block: rows of this many floats (8 beyond a multiple of 32: eight heads' pairs lie in different banks)
__host__ __device__ constexpr int paged_pitch(int span) { return (span + 31) / 32 * 32 + 8; }
template <class Core> size_t paged_fused_bytes(int span)
{
    const size_t work = (size_t)span * 8 + (size_t)Core::HEADS * paged_pitch(span) * 4;
    return work > paged_out_bytes<Core>() ? work : paged_out_bytes<Core>();
}
template <class Core> size_t paged_values_bytes(int span)
{
    return (size_t)span * 8 > paged_out_bytes<Core>() ? (size_t)span * 8 : paged_out_bytes<Core>();
}

#define NM_PAGED_EXP_TABLE()                                                                             \
    __shared__ float2 s_exp[NM_MAX_SEGMENTS];                                                            \
    for (int i = threadIdx.x; i < a.exp_tab->n; i += PAGED_THREADS) s_exp[i] = a.exp_tab->kb[i];         \
    const PagedExp exp = {s_exp, a.exp_tab->inv_h, a.exp_tab->off, (float)(a.exp_tab->n - 1)}

// One launch: a cluster per unit, its blocks sharing the row's tokens evenly.
template <class Core>
__global__ void __launch_bounds__(PAGED_THREADS, 2) paged_fused_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    extern __shared__ __align__(128) unsigned char paged_smem[];
    __shared__ float s_max[PAGED_WARPS][Core::HEADS], s_cluster_max[8][Core::HEADS], s_row_max[Core::HEADS];
    __shared__ float s_sum[PAGED_WARPS][Core::HEADS], s_block_sum[Core::HEADS];
    NM_PAGED_EXP_TABLE();
    uint32_t ctas;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const int rank = (int)nm_cluster_ctarank();
    const PagedUnit u = paged_unit<Core>(a, blockIdx.x / ctas);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, u.b);
    if (len < 0) return;   // the whole cluster
    const int per = ((len + (int)ctas - 1) / (int)ctas + 15) / 16 * 16, first = min(len, rank * per), count = min(len - first, per);
    int64_t* off = reinterpret_cast<int64_t*>(paged_smem);
    float* sc = reinterpret_cast<float*>(paged_smem + (size_t)a.span * 8);
    const int pitch = paged_pitch(a.span), warp = threadIdx.x >> 5;
    paged_offsets(a, u.b, first, count, off);
    __syncthreads();
    Core::scores(a, (const T*)a.d.Q + (int64_t)u.b * a.d.ld_q + (int64_t)u.h0 * a.d.d, u.nh, (const T*)a.d.k_cache + (int64_t)u.kv * a.d.stride_head,
                 off, count, s_max[warp], [&](int h, int i, float s) { sc[h * pitch + i] = s; });
    Core core;
    float* out = reinterpret_cast<float*>(paged_smem);
    core.values(
        a, u.nh, (const T*)a.d.v_cache + (int64_t)u.kv * a.d.stride_head, off, count, exp, s_sum[warp], out + warp * (Core::HEADS * Core::D),
        [&] {   // the row's maxima
            __syncthreads();
            if (threadIdx.x < Core::HEADS) {
                float x = s_max[0][threadIdx.x];
                for (int w = 1; w < PAGED_WARPS; ++w) x = fmaxf(x, s_max[w][threadIdx.x]);
                if (ctas == 1) {
                    s_row_max[threadIdx.x] = x;
                } else {
                    const uint32_t at = nm_smem_u32(&s_cluster_max[rank][threadIdx.x]);
                    for (uint32_t c = 0; c < ctas; ++c)
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(nm_mapa(at, c)), "f"(x) : "memory");
                }
            }
            if (ctas > 1) {
                nm_cluster_sync();
                if (threadIdx.x < Core::HEADS) {
                    float x = s_cluster_max[0][threadIdx.x];
                    for (uint32_t c = 1; c < ctas; ++c) x = fmaxf(x, s_cluster_max[c][threadIdx.x]);
                    s_row_max[threadIdx.x] = x;
                }
            }
            __syncthreads();
            return (const float*)s_row_max;
        },
        [&](int h, int i) { return *reinterpret_cast<const float2*>(sc + h * pitch + i); });
    __syncthreads();
    // the block's sums in warp 0's place
    for (int x = threadIdx.x; x < u.nh * Core::D; x += PAGED_THREADS) {
        float o = out[x];
        for (int w = 1; w < PAGED_WARPS; ++w) o += out[w * (Core::HEADS * Core::D) + x];
        out[x] = o;
    }
    if (threadIdx.x < Core::HEADS) {
        float s = s_sum[0][threadIdx.x];
        for (int w = 1; w < PAGED_WARPS; ++w) s += s_sum[w][threadIdx.x];
        s_block_sum[threadIdx.x] = s;
    }
    if (ctas > 1) nm_cluster_sync();
    else __syncthreads();
    for (int x = rank * PAGED_THREADS + threadIdx.x; x < u.nh * Core::D; x += (int)ctas * PAGED_THREADS) {
        const int h = x / Core::D, c = x - h * Core::D;
        if (c >= a.d.d) continue;
        float o = 0.f, s = 0.f;
        for (uint32_t r = 0; r < ctas; ++r) {
            float po, ps;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(po) : "r"(nm_mapa(nm_smem_u32(out + x), r)) : "memory");
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(ps) : "r"(nm_mapa(nm_smem_u32(&s_block_sum[h]), r)) : "memory");
            o += po;
            s += ps;
        }
        ((T*)a.d.out)[(int64_t)u.b * a.d.ld_out + (int64_t)(u.h0 + h) * a.d.d + c] = NmType<T>::from_f(len ? o * paged_table(a.recip_tab, s) : 0.f);
    }
    if (ctas > 1) nm_cluster_sync();   // no block leaves while another reads its shared memory
}

template <class Core>
__global__ void __launch_bounds__(PAGED_THREADS, 2) paged_scores_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    extern __shared__ __align__(128) unsigned char paged_smem[];
    __shared__ float s_max[PAGED_WARPS][Core::HEADS];
    const int span = (int)(blockIdx.x % a.spans), first = span * a.span;
    const PagedUnit u = paged_unit<Core>(a, blockIdx.x / a.spans);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, u.b);
    if (first >= len) return;
    const int count = min(len - first, a.span);
    int64_t* off = reinterpret_cast<int64_t*>(paged_smem);
    paged_offsets(a, u.b, first, count, off);
    __syncthreads();
    float* sc = a.scores + ((int64_t)u.b * a.d.heads + u.h0) * a.row + first;
    Core::scores(a, (const T*)a.d.Q + (int64_t)u.b * a.d.ld_q + (int64_t)u.h0 * a.d.d, u.nh, (const T*)a.d.k_cache + (int64_t)u.kv * a.d.stride_head,
                 off, count, s_max[threadIdx.x >> 5], [&](int h, int i, float s) {
                     if (h < u.nh) sc[h * a.row + i] = s;
                 });
    __syncthreads();
    if ((int)threadIdx.x < u.nh) {
        float x = s_max[0][threadIdx.x];
        for (int w = 1; w < PAGED_WARPS; ++w) x = fmaxf(x, s_max[w][threadIdx.x]);
        a.maxima[((int64_t)u.b * a.d.heads + u.h0 + threadIdx.x) * a.spans + span] = x;
    }
}

template <class Core>
__global__ void __launch_bounds__(PAGED_THREADS, 2) paged_values_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    extern __shared__ __align__(128) unsigned char paged_smem[];
    __shared__ float s_m[Core::HEADS], s_sum[PAGED_WARPS][Core::HEADS];
    NM_PAGED_EXP_TABLE();
    const int span = (int)(blockIdx.x % a.spans), first = span * a.span, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const PagedUnit u = paged_unit<Core>(a, blockIdx.x / a.spans);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, u.b);
    if (first >= len) return;
    const int count = min(len - first, a.span), used = (len + a.span - 1) / a.span;
    int64_t* off = reinterpret_cast<int64_t*>(paged_smem);
    paged_offsets(a, u.b, first, count, off);
    const int64_t head0 = (int64_t)u.b * a.d.heads + u.h0;
    for (int h = warp; h < Core::HEADS; h += PAGED_WARPS) {
        float m = -INFINITY;
        if (h < u.nh)
            for (int i = lane; i < used; i += 32) m = fmaxf(m, a.maxima[(head0 + h) * a.spans + i]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) s_m[h] = m;
    }
    __syncthreads();
    const float* sc = a.scores + head0 * a.row + first;
    Core core;
    float* out = reinterpret_cast<float*>(paged_smem);
    core.values(a, u.nh, (const T*)a.d.v_cache + (int64_t)u.kv * a.d.stride_head, off, count, exp, s_sum[warp], out + warp * (Core::HEADS * Core::D),
                [&] { return (const float*)s_m; }, [&](int h, int i) { return *reinterpret_cast<const float2*>(sc + h * a.row + i); });
    __syncthreads();
    for (int x = threadIdx.x; x < u.nh * Core::D; x += PAGED_THREADS) {
        const int h = x / Core::D, c = x - h * Core::D;
        if (c >= a.d.d) continue;
        float o = out[x], s = s_sum[0][h];
        for (int w = 1; w < PAGED_WARPS; ++w) {
            o += out[w * (Core::HEADS * Core::D) + x];
            s += s_sum[w][h];
        }
        const int64_t row = (head0 + h) * a.spans + span;
        a.outs[row * a.d.d + c] = o;
        if (c == 0) a.sums[row] = s;
    }
}

// A block per request and head.
template <typename T>
__global__ void __launch_bounds__(128) paged_join_kernel(const PagedArgs a)
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
    for (int c = threadIdx.x; c < a.d.d; c += 128) {
        float o = 0.f;
        for (int i = 0; i < used; ++i) o += a.outs[(bh * a.spans + i) * a.d.d + c];
        ((T*)a.d.out)[(int64_t)b * a.d.ld_out + (int64_t)h * a.d.d + c] = NmType<T>::from_f(used ? o * r : 0.f);
    }
}

// ---------------------------------------------------------------- host

constexpr int PAGED_SMS = 148;   // the layout must not depend on the device: the workspace's size is asked for without one

// Query heads of a unit: 16 where the tensor cores take them and the registers hold their sums, otherwise as few as cover the group.
int paged_heads(const nm_attn_paged_desc* d, bool mma)
{
    const int group = d->heads / d->kv_heads;
    if (mma) return group > 8 && d->d <= 128 ? 16 : 8;
    return group >= 8 ? 8 : group >= 4 ? 4 : group >= 2 ? 2 : 1;
}
bool paged_mma_supported(const nm_attn_paged_desc* d) { return d->dtype != NM_F32 && (d->d == 64 || d->d == 96 || d->d == 128 || d->d == 256); }

struct PagedLayout {
    bool mma, fused;
    int heads, blocks_per_head, ctas, span, spans;
    int64_t units, row;
    size_t scores, maxima, sums, outs, total;
};
PagedLayout layout_of(const nm_attn_paged_desc* d)
{
    PagedLayout l;
    const int group = d->heads / d->kv_heads;
    l.mma = paged_mma_supported(d);
    l.heads = paged_heads(d, l.mma);
    l.blocks_per_head = (group + l.heads - 1) / l.heads;
    l.units = (int64_t)d->B * d->kv_heads * l.blocks_per_head;
    l.scores = l.maxima = l.sums = l.outs = l.total = 0;
    l.row = 0;
    l.spans = 1;
    const int cap = l.heads == 16 ? 1024 : 2048;   // two blocks an SM
    l.fused = d->max_len <= 8 * cap;
    if (l.fused) {
        int ctas = 1;
        while (ctas < 8 && ((d->max_len + ctas - 1) / ctas > cap || (l.units * ctas * 2 <= 2 * PAGED_SMS && d->max_len > ctas * 128))) ctas *= 2;
        l.ctas = ctas;
        l.span = ((d->max_len + ctas - 1) / ctas + 15) / 16 * 16;
        return l;
    }
    l.ctas = 1;
    // spans of whole 128 tokens, as many as make twelve blocks per SM
    const int64_t tokens = (l.units * d->max_len + PAGED_SMS * 12 - 1) / (PAGED_SMS * 12);
    l.span = (int)(((tokens > 2048 ? 2048 : tokens) + 127) / 128 * 128);
    l.spans = (int)(((int64_t)d->max_len + l.span - 1) / l.span);
    l.row = ((int64_t)d->max_len + 31) / 32 * 32;
    const size_t bh = (size_t)d->B * d->heads;
    auto take = [&l](size_t bytes) { const size_t at = l.total; l.total += (bytes + 255) / 256 * 256; return at; };
    l.scores = take(bh * l.row * 4);
    l.maxima = take(bh * l.spans * 4);
    l.sums = take(bh * l.spans * 4);
    l.outs = take(bh * l.spans * d->d * 4);
    return l;
}

template <typename K>
nm_status paged_launch(nm_ctx* ctx, K kernel, const PagedArgs& a, int64_t blocks, int threads, size_t smem, int ctas, double bytes, cudaStream_t st)
{
    if (blocks > INT32_MAX) return NM_ERR_SHAPE;
    // (48 KB are there without asking, the kernels' static arrays among them)
    if (smem > 40 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return NM_ERR_CUDA;
    NmLaunchScope scope(ctx, NM_KERNEL_ATTENTION_PAGED, bytes, st);
    NmLaunchConfig lc(ctx, dim3((unsigned)blocks), threads, smem, st, ctas);
    return cudaLaunchKernelEx(&lc.cfg, kernel, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

template <class Core>
nm_status launch(nm_ctx* ctx, const PagedArgs& a, const PagedLayout& l, cudaStream_t st)
{
    using T = typename Core::Elem;
    const double bytes = (double)a.d.B * a.d.max_len * a.d.kv_heads * a.d.d * sizeof(T);
    if (l.fused) return paged_launch(ctx, paged_fused_kernel<Core>, a, l.units * l.ctas, PAGED_THREADS, paged_fused_bytes<Core>(l.span), l.ctas, 2 * bytes, st);
    nm_status s = paged_launch(ctx, paged_scores_kernel<Core>, a, l.units * l.spans, PAGED_THREADS, (size_t)l.span * 8, 1, bytes, st);
    if (s != NM_OK) return s;
    s = paged_launch(ctx, paged_values_kernel<Core>, a, l.units * l.spans, PAGED_THREADS, paged_values_bytes<Core>(l.span), 1, bytes, st);
    if (s != NM_OK) return s;
    return paged_launch(ctx, paged_join_kernel<T>, a, (int64_t)a.d.B * a.d.heads, 128, 0, 1, 0.0, st);
}

template <typename T>
nm_status dispatch(nm_ctx* ctx, const PagedArgs& a, const PagedLayout& l, cudaStream_t st)
{
    if constexpr (sizeof(T) == 2) {
        if (l.mma) {
            const bool two = l.heads == 16;
            switch (a.d.d) {
            case 64: return two ? launch<PagedMma<T, 64, 2>>(ctx, a, l, st) : launch<PagedMma<T, 64, 1>>(ctx, a, l, st);
            case 96: return two ? launch<PagedMma<T, 96, 2>>(ctx, a, l, st) : launch<PagedMma<T, 96, 1>>(ctx, a, l, st);
            case 128: return two ? launch<PagedMma<T, 128, 2>>(ctx, a, l, st) : launch<PagedMma<T, 128, 1>>(ctx, a, l, st);
            default: return launch<PagedMma<T, 256, 1>>(ctx, a, l, st);
            }
        }
    }
    const int vecs = a.d.d * (int)sizeof(T) / 16;
#define NM_PAGED_HB(LPK, VPL)                                                          \
    do {                                                                               \
        if (l.heads == 8) return launch<PagedFma<T, LPK, VPL, 8>>(ctx, a, l, st);      \
        if (l.heads == 4) return launch<PagedFma<T, LPK, VPL, 4>>(ctx, a, l, st);      \
        if (l.heads == 2) return launch<PagedFma<T, LPK, VPL, 2>>(ctx, a, l, st);      \
        return launch<PagedFma<T, LPK, VPL, 1>>(ctx, a, l, st);                        \
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
    switch (d->dtype) {
    case NM_F32: return dispatch<float>(ctx, a, l, st);
    case NM_BF16: return dispatch<__nv_bfloat16>(ctx, a, l, st);
    case NM_F16: return dispatch<__half>(ctx, a, l, st);
    default: return NM_ERR_UNSUPPORTED;
    }
}
