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

#ifndef RINGB
#define RINGB 8192
#endif
constexpr int PAGED_WARPS = 8, PAGED_THREADS = PAGED_WARPS * 32, PAGED_RING = RINGB;   // bytes of a warp's ring

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

// Asynchronous copies: a warp copies what it will read itself, so its tiles need no barrier of the block.  Invalid tokens are filled
// with zeros.
__device__ __forceinline__ void paged_copy(uint32_t dst, const void* src, bool valid)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void paged_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void paged_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Runs a warp's tiles through its ring: fetch(i0, stage) starts the copies of the tile at token i0, use(i0, stage) consumes it.  `ready` is
// called once the first tiles are on their way.
template <int STAGES, int TILE, typename Fetch, typename Ready, typename Use>
__device__ __forceinline__ void paged_pipeline(int count, Fetch fetch, Ready ready, Use use)
{
    constexpr int STEP = PAGED_WARPS * TILE;
    int i0 = (threadIdx.x >> 5) * TILE, next = i0, stage = 0;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s, next += STEP) {
        if (next < count) fetch(next, s);
        paged_commit();
    }
    ready();
    for (; i0 < count; i0 += STEP, next += STEP) {
        if (next < count) fetch(next, stage == 0 ? STAGES - 1 : stage - 1);   // the stage that the tile before has left
        paged_commit();
        paged_wait<STAGES - 1>();
        __syncwarp();   // the lanes' copies are there
        use(i0, stage);
        __syncwarp();   // and have been read
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    paged_wait<0>();
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

// Four 8 x 8 matrices of 16-bit numbers, lane l giving the address of row l % 8 of matrix l / 8; transposed on request.
__device__ __forceinline__ void paged_ldmatrix(uint32_t* r, uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void paged_ldmatrix_trans(uint32_t* r, uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}

// Tiles of 16 tokens, NT tiles of 8 query heads: S^T = K Q^T and O^T = V^T P^T, tokens or channels as rows, so that eight heads fill
// a product.  Rows are copied whole (fragments loaded from the cache directly would take 64 bytes of a row at a time: 2.9 to 4.9 TB/s
// where whole rows reach ...) and lie in the ring with their 16-byte pieces permuted, piece c of row r at c ^ (r & 7)
// (rows of 96 channels one piece apart instead): neither the copies nor the matrix reads collide.
// Probabilities are two 16-bit terms.
template <typename T, int D_, int NT> struct PagedMma {
    using Elem = T;
    static constexpr int D = D_, HEADS = NT * 8, TILE = 16, LANES = D / 8;   // lanes of a row
    static constexpr bool POW2 = (LANES & (LANES - 1)) == 0;
    static constexpr int PITCH = D * 2 + (POW2 ? 0 : 16), STAGE = TILE * PITCH, STAGES = PAGED_RING / STAGE < 2 ? 2 : PAGED_RING / STAGE, RING = STAGES * STAGE;   // bytes of a warp
    static_assert(D % 32 == 0 && HEADS * D * 4 <= RING, "whole 32-channel pieces; a warp's sums fit its ring");
    static __device__ __forceinline__ float2 read(const float* s) { return *reinterpret_cast<const float2*>(s); }   // two tokens' scores

    static __device__ __forceinline__ uint32_t piece(int row, int c) { return row * PITCH + ((POW2 ? c ^ (row & 7) : c) << 4); }
    static __device__ __forceinline__ void fetch(const T* base, const int64_t* off, int count, uint32_t ring_at, int i0, int stage)
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int x = 0; x < TILE * LANES / 32; ++x) {
            const int at = x * 32 + lane, row = at / LANES, c = at % LANES, i = i0 + row;
            const int64_t o = i < count ? off[i] : -1;
            paged_copy(ring_at + stage * STAGE + piece(row, c), o >= 0 ? base + o + c * 8 : base, o >= 0);
        }
    }

    // put(h, i, s) takes the score of head h and token i; the heads' maxima over the warp's tokens go to warp_max
    template <typename Put>
    static __device__ __forceinline__ void scores(const PagedArgs& a, const T* Q, int nh, const T* K, const int64_t* off, int count, unsigned char* ring,
                                                  float* warp_max, Put put)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        const uint32_t ring_at = nm_smem_u32(ring);
        uint32_t q[NT][D / 16][2];
        float m[NT][2];
        paged_pipeline<STAGES, TILE>(
            count, [&](int i0, int stage) { fetch(K, off, count, ring_at, i0, stage); },
            [&] {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    m[n][0] = m[n][1] = -INFINITY;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            q[n][c][r] = n * 8 + g < nh ? *reinterpret_cast<const uint32_t*>(Q + (n * 8 + g) * D + c * 16 + r * 8 + t * 2) : 0;
                }
            },
            [&](int i0, int stage) {
                float s[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
                const uint32_t tile = ring_at + stage * STAGE;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t k[4];
                    paged_ldmatrix(k, tile + piece(lane & 15, 2 * c + (lane >> 4)));
#pragma unroll
                    for (int n = 0; n < NT; ++n) paged_mma(s[n], k[0], k[1], k[2], k[3], q[n][c][0], q[n][c][1], T());
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float v = s[n][r] * a.d.scale;
                        const int j = i0 + g + (r >> 1) * 8;
                        if (j < count) {
                            m[n][r & 1] = fmaxf(m[n][r & 1], v);
                            put(n * 8 + 2 * t + (r & 1), j, v);
                        }
                    }
            });
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) m[n][r] = fmaxf(m[n][r], __shfl_xor_sync(0xffffffffu, m[n][r], o));
                if (g == 0) warp_max[n * 8 + 2 * t + r] = m[n][r];
            }
    }

    // get(h, i) reads the scores of head h and tokens i, i + 1; `maxima` is called once the first tiles are on their way.  The warp's
    // sums go to warp_sum and, as [head][channel], to the ring.
    template <typename Max, typename Get>
    static __device__ __forceinline__ void values(const PagedArgs& a, int nh, const T* V, const int64_t* off, int count, PagedExp exp, unsigned char* ring,
                                                  float* warp_sum, Max maxima, Get get)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        const uint32_t ring_at = nm_smem_u32(ring);
        float acc[NT][D / 16][4], sum[NT], m[NT];
        paged_pipeline<STAGES, TILE>(
            count, [&](int i0, int stage) { fetch(V, off, count, ring_at, i0, stage); },
            [&] {
                const float* x = maxima();
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    m[n] = x[n * 8 + g];
                    sum[n] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) acc[n][c][0] = acc[n][c][1] = acc[n][c][2] = acc[n][c][3] = 0.f;
                }
            },
            [&](int i0, int stage) {
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
                const uint32_t tile = ring_at + stage * STAGE;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t v[4];   // channels c * 16 + 0..7 and 8..15 of tokens 0..7, then of tokens 8..15
                    paged_ldmatrix_trans(v, tile + piece((lane & 7) + (lane >> 4) * 8, 2 * c + ((lane >> 3) & 1)));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        paged_mma(acc[n][c], v[0], v[1], v[2], v[3], hi[n][0], hi[n][1], T());
                        paged_mma(acc[n][c], v[0], v[1], v[2], v[3], lo[n][0], lo[n][1], T());
                    }
                }
            });
        __syncwarp();   // the ring has been read
        float* out = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
            sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
            if (t == 0) warp_sum[n * 8 + g] = sum[n];
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) out[(n * 8 + 2 * t + (r & 1)) * D + c * 16 + g + (r >> 1) * 8] = acc[n][c][r];
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

// Sums each of v[0..COUNT-1] over the LPK lanes of a token; lane `part` of them is left with sum number first(part) .. + LEFT - 1 in
// v[0..LEFT-1].  While there are several sums a step halves their number (each lane passes on the half that the other lane keeps),
// so COUNT sums take COUNT - 1 shuffles, not COUNT * log2(LPK).
template <int COUNT, int LPK> struct PagedSums {
    static constexpr int LEFT = COUNT > LPK ? COUNT / LPK : 1;
    static __device__ __forceinline__ void reduce(float* v, int part)
    {
        int n = COUNT;
#pragma unroll
        for (int o = LPK / 2; o > 0; o >>= 1) {
            if (n > 1) {
                n >>= 1;
                const bool upper = part & o;
#pragma unroll
                for (int i = 0; i < COUNT / 2; ++i)
                    if (i < n) {
                        const float keep = upper ? v[i + n] : v[i], give = upper ? v[i] : v[i + n];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                    }
            } else {
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
            }
        }
    }
    // number of the first sum that lane `part` has
    static __device__ __forceinline__ int first(int part)
    {
        int at = 0, n = COUNT;
#pragma unroll
        for (int o = LPK / 2; o > 0; o >>= 1)
            if (n > 1) {
                n >>= 1;
                at += part & o ? n : 0;
            }
        return at;
    }
    // whether the lane is the one of those with the same sums that writes them
    static __device__ __forceinline__ bool writes(int part) { return COUNT >= LPK || (part & (LPK / COUNT - 1)) == 0; }
};

// LPK lanes hold a token, VPL vectors of 16 bytes each (lanes behind the head's channels hold none), U tokens one after another:
// tiles of U * 32/LPK tokens against HB query heads in registers.
template <typename T, int LPK, int VPL, int HB> struct PagedFma {
    using Elem = T;
    static constexpr int N = Vec16<T>::N, U = 4, SUB = 32 / LPK, TILE = U * SUB, HEADS = HB, D = LPK * VPL * N;   // D: room for the channels
    static constexpr int STAGE = U * VPL * 512, STAGES = PAGED_RING / STAGE, RING = STAGES * STAGE;
    static_assert(HEADS * D * 4 <= RING, "a warp's sums fit its ring");
    static __device__ __forceinline__ float read(const float* s) { return *s; }

    static __device__ __forceinline__ void fetch(const PagedArgs& a, const T* base, const int64_t* off, int count, uint32_t ring_at, int i0, int stage)
    {
        const int lane = threadIdx.x & 31, part = lane & (LPK - 1), sub = lane / LPK;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + k * SUB + sub;
            const int64_t at = i < count ? off[i] : -1;
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const int c = (v * LPK + part) * N;
                const bool valid = at >= 0 && c < a.d.d;
                paged_copy(ring_at + stage * STAGE + (k * VPL + v) * 512 + lane * 16, valid ? base + at + c : base, valid);
            }
        }
    }

    template <typename Put>
    static __device__ __forceinline__ void scores(const PagedArgs& a, const T* Q, int nh, const T* K, const int64_t* off, int count, unsigned char* ring,
                                                  float* warp_max, Put put)
    {
        using Sums = PagedSums<HB * U, LPK>;   // sum number k * HB + h: token k, head h
        const int lane = threadIdx.x & 31, part = lane & (LPK - 1), sub = lane / LPK;
        const uint32_t ring_at = nm_smem_u32(ring);
        const int sum0 = Sums::first(part);
        float q[HB][VPL][N], m[Sums::LEFT];
        paged_pipeline<STAGES, TILE>(
            count, [&](int i0, int stage) { fetch(a, K, off, count, ring_at, i0, stage); },
            [&] {
#pragma unroll
                for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        const int c = (v * LPK + part) * N;
                        Vec16<T> x;
                        x.raw = h < nh && c < a.d.d ? *reinterpret_cast<const uint4*>(Q + h * a.d.d + c) : make_uint4(0, 0, 0, 0);
                        x.get(q[h][v]);
                    }
#pragma unroll
                for (int i = 0; i < Sums::LEFT; ++i) m[i] = -INFINITY;
            },
            [&](int i0, int stage) {
                const uint4* tile = reinterpret_cast<const uint4*>(ring + stage * STAGE) + lane;
                float dot[HB * U];
#pragma unroll
                for (int k = 0; k < U; ++k) {
#pragma unroll
                    for (int h = 0; h < HB; ++h) dot[k * HB + h] = 0.f;
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        Vec16<T> x;
                        x.raw = tile[(k * VPL + v) * 32];
                        float f[N];
                        x.get(f);
#pragma unroll
                        for (int h = 0; h < HB; ++h)
#pragma unroll
                            for (int e = 0; e < N; ++e) dot[k * HB + h] = __fmaf_rn(q[h][v][e], f[e], dot[k * HB + h]);
                    }
                }
                Sums::reduce(dot, part);
#pragma unroll
                for (int l = 0; l < Sums::LEFT; ++l) {
                    const int h = (sum0 + l) % HB, i = i0 + (sum0 + l) / HB * SUB + sub;
                    const float s = dot[l] * a.d.scale;
                    if (i < count && h < nh) {
                        m[l] = fmaxf(m[l], s);
                        if (Sums::writes(part)) put(h, i, s);
                    }
                }
            });
        // a head's maximum: over the lanes (and places) with sums of this head
#pragma unroll
        for (int h = 0; h < HB; ++h) {
            float x = -INFINITY;
#pragma unroll
            for (int l = 0; l < Sums::LEFT; ++l) x = (sum0 + l) % HB == h ? fmaxf(x, m[l]) : x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            if (lane == 0) warp_max[h] = x;
        }
    }

    template <typename Max, typename Get>
    static __device__ __forceinline__ void values(const PagedArgs& a, int nh, const T* V, const int64_t* off, int count, PagedExp exp, unsigned char* ring,
                                                  float* warp_sum, Max maxima, Get get)
    {
        const int lane = threadIdx.x & 31, part = lane & (LPK - 1), sub = lane / LPK;
        const uint32_t ring_at = nm_smem_u32(ring);
        constexpr int TH = U * HB;   // a token's exponentials are shared by its lanes: lane `part` computes number part, part + LPK, ...
        constexpr int MINE = (TH + LPK - 1) / LPK;
        float acc[HB][VPL][N], sum[MINE], m[MINE];
        paged_pipeline<STAGES, TILE>(
            count, [&](int i0, int stage) { fetch(a, V, off, count, ring_at, i0, stage); },
            [&] {
                const float* x = maxima();
#pragma unroll
                for (int l = 0; l < MINE; ++l) {
                    m[l] = x[(l * LPK + part) % HB];
                    sum[l] = 0.f;
                }
#pragma unroll
                for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int v = 0; v < VPL; ++v)
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[h][v][e] = 0.f;
            },
            [&](int i0, int stage) {
                const uint4* tile = reinterpret_cast<const uint4*>(ring + stage * STAGE) + lane;
                float mine[MINE];
#pragma unroll
                for (int l = 0; l < MINE; ++l) {
                    const int x = l * LPK + part, h = x % HB, i = i0 + x / HB * SUB + sub;
                    mine[l] = x < TH && h < nh && i < count ? exp(get(h, i) - m[l]) : 0.f;
                    sum[l] += mine[l];
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    float e[HB];
#pragma unroll
                    for (int h = 0; h < HB; ++h)
                        e[h] = __shfl_sync(0xffffffffu, mine[(k * HB + h) / LPK], (lane & ~(LPK - 1)) | ((k * HB + h) % LPK));
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        Vec16<T> x;
                        x.raw = tile[(k * VPL + v) * 32];
                        float f[N];
                        x.get(f);
#pragma unroll
                        for (int h = 0; h < HB; ++h)
#pragma unroll
                            for (int c = 0; c < N; ++c) acc[h][v][c] = __fmaf_rn(e[h], f[c], acc[h][v][c]);
                    }
                }
            });
        __syncwarp();   // the ring has been read
        float* out = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int h = 0; h < HB; ++h) {
            float s = 0.f;
#pragma unroll
            for (int l = 0; l < MINE; ++l) s += (l * LPK + part) % HB == h ? sum[l] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0) warp_sum[h] = s;
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
#pragma unroll
                for (int c = 0; c < N; ++c) {
#pragma unroll
                    for (int o = 16; o >= LPK; o >>= 1) acc[h][v][c] += __shfl_xor_sync(0xffffffffu, acc[h][v][c], o);
                    if (sub == 0) out[h * D + (v * LPK + part) * N + c] = acc[h][v][c];
                }
            }
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
// scores of a block: rows of this many floats (8 beyond a multiple of 32: eight heads' pairs lie in different banks)
__host__ __device__ constexpr int paged_pitch(int span) { return (span + 31) / 32 * 32 + 8; }
template <class Core> constexpr size_t paged_split_bytes(int span) { return (size_t)PAGED_WARPS * Core::RING + (size_t)span * 8; }
template <class Core> constexpr size_t paged_fused_bytes(int span)
{
    return paged_split_bytes<Core>(span) + (size_t)Core::HEADS * paged_pitch(span) * 4;
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
    const int pitch = paged_pitch(a.span), warp = threadIdx.x >> 5;
    unsigned char* ring = paged_smem + warp * Core::RING;
    int64_t* off = reinterpret_cast<int64_t*>(paged_smem + PAGED_WARPS * Core::RING);
    float* sc = reinterpret_cast<float*>(off + a.span);
    paged_offsets(a, u.b, first, count, off);
    __syncthreads();
    Core::scores(a, (const T*)a.d.Q + (int64_t)u.b * a.d.ld_q + (int64_t)u.h0 * a.d.d, u.nh, (const T*)a.d.k_cache + (int64_t)u.kv * a.d.stride_head,
                 off, count, ring, s_max[warp], [&](int h, int i, float s) { sc[h * pitch + i] = s; });
    Core::values(
        a, u.nh, (const T*)a.d.v_cache + (int64_t)u.kv * a.d.stride_head, off, count, exp, ring, s_sum[warp],
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
        [&](int h, int i) { return Core::read(sc + h * pitch + i); });
    __syncthreads();
    // the block's sums in warp 0's place
    float* out = reinterpret_cast<float*>(paged_smem);
    for (int x = threadIdx.x; x < u.nh * Core::D; x += PAGED_THREADS) {
        float o = out[x];
        for (int w = 1; w < PAGED_WARPS; ++w) o += out[w * (Core::RING / 4) + x];
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
    unsigned char* ring = paged_smem + (threadIdx.x >> 5) * Core::RING;
    int64_t* off = reinterpret_cast<int64_t*>(paged_smem + PAGED_WARPS * Core::RING);
    paged_offsets(a, u.b, first, count, off);
    __syncthreads();
    float* sc = a.scores + ((int64_t)u.b * a.d.heads + u.h0) * a.row + first;
    Core::scores(a, (const T*)a.d.Q + (int64_t)u.b * a.d.ld_q + (int64_t)u.h0 * a.d.d, u.nh, (const T*)a.d.k_cache + (int64_t)u.kv * a.d.stride_head,
                 off, count, ring, s_max[threadIdx.x >> 5], [&](int h, int i, float s) {
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
    unsigned char* ring = paged_smem + warp * Core::RING;
    int64_t* off = reinterpret_cast<int64_t*>(paged_smem + PAGED_WARPS * Core::RING);
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
    Core::values(a, u.nh, (const T*)a.d.v_cache + (int64_t)u.kv * a.d.stride_head, off, count, exp, ring, s_sum[warp], [&] { return (const float*)s_m; },
                 [&](int h, int i) { return Core::read(sc + h * a.row + i); });
    __syncthreads();
    for (int x = threadIdx.x; x < u.nh * Core::D; x += PAGED_THREADS) {
        const int h = x / Core::D, c = x - h * Core::D;
        if (c >= a.d.d) continue;
        const float* out = reinterpret_cast<const float*>(paged_smem);
        float o = out[x], s = s_sum[0][h];
        for (int w = 1; w < PAGED_WARPS; ++w) {
            o += out[w * (Core::RING / 4) + x];
            s += s_sum[w][h];
        }
        const int64_t row = (head0 + h) * a.spans + span;
        a.outs[row * a.d.d + c] = o;
        if (c == 0) a.sums[row] = s;
    }
}

// A block per request and head: four warps take every fourth span, a lane four channels of a span.
constexpr int JOIN_WARPS = 4;
template <typename T>
__global__ void __launch_bounds__(JOIN_WARPS * 32) paged_join_kernel(const PagedArgs a)
{
    __shared__ float s_out[JOIN_WARPS][256], s_sum[JOIN_WARPS];
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.d.heads), h = (int)(bh - (int64_t)b * a.d.heads), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const int len = paged_length(a, b);
    if (len < 0) return;
    const int used = (len + a.span - 1) / a.span;
    float s = 0.f;
    for (int i = warp * 32 + lane; i < used; i += JOIN_WARPS * 32) s += a.sums[bh * a.spans + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) s_sum[warp] = s;
    for (int c = lane * 4; c < a.d.d; c += 128) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = warp; i < used; i += JOIN_WARPS) {
            const float4 v = *reinterpret_cast<const float4*>(a.outs + (bh * a.spans + i) * a.d.d + c);
            o.x += v.x;
            o.y += v.y;
            o.z += v.z;
            o.w += v.w;
        }
        *reinterpret_cast<float4*>(&s_out[warp][c]) = o;
    }
    __syncthreads();
    s = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
    const float r = paged_table(a.recip_tab, s);
    for (int c = threadIdx.x; c < a.d.d; c += JOIN_WARPS * 32) {
        const float o = s_out[0][c] + s_out[1][c] + s_out[2][c] + s_out[3][c];
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
// Tokens of a block of the fused form: offsets and scores take what rings of 64 KB leave of half an SM's shared memory.
int paged_cap(int heads) { return (44 * 1024 - heads * 4 * 40) / (8 + heads * 4) / 16 * 16; }
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
    const int cap = paged_cap(l.heads);
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
    nm_status s = paged_launch(ctx, paged_scores_kernel<Core>, a, l.units * l.spans, PAGED_THREADS, paged_split_bytes<Core>(l.span), 1, bytes, st);
    if (s != NM_OK) return s;
    s = paged_launch(ctx, paged_values_kernel<Core>, a, l.units * l.spans, PAGED_THREADS, paged_split_bytes<Core>(l.span), 1, bytes, st);
    if (s != NM_OK) return s;
    return paged_launch(ctx, paged_join_kernel<T>, a, (int64_t)a.d.B * a.d.heads, JOIN_WARPS * 32, 0, 1, 0.0, st);
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
