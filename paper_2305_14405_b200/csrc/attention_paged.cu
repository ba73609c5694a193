// Attention of one new token per request over a paged key-value cache with PWL softmax.  Bound by the bytes of K and V.
//
// A PWL exponential is not multiplicative, so e_j = PWL_exp(s_j - m) needs the maximum m of the whole row before the first value is
// weighted: a running maximum that rescales earlier sums would compute another function.  Keys and values are still read once
// each, because the scores are kept (4 bytes per token and query head, against 2 d elements of K and V per token and key head).
// A unit of work is a request, a key head and up to HEADS of its query heads.
//   fused   one launch: a cluster of blocks per unit, scores in shared memory, maxima and sums exchanged within the cluster
//   split   two launches, scores in the workspace: all units' tokens lie one after another and every block takes an equal share, so
//           that requests of any lengths keep all SMs busy to the end; a unit that several blocks have is joined by the last of them,
//           or, if there are few units and so many blocks each, by a third launch
// A block's tokens are split over its warps in tiles.  Two cores do a tile:
//   PagedMma   16-bit types, d a multiple of 32: m16n8k16 products
//   PagedFma   fp32 and other d: FMAs, a few lanes per token
// Partial sums are fp32 and are added in the order of warps and blocks: results do not depend on timing.
// Measured: bf16, 48 requests of up to 8192 tokens, 8 key heads of 128 channels (697 MB) 129 us, 5.4 TB/s; one of 131071 tokens (537 MB)
// 103 us, 5.2 TB/s; 12 heads of 64 over 500 tokens 5.7 us, the latency of a chain (pages, keys, maximum, values, sums) and a launch.
// Of the long rows the scores kernel is near the bytes' time; the values kernel waits for it, and the sums' join, are the rest.  In between
// (10 to 150 MB) the fixed costs count most: 15 requests of up to 2898 tokens (95 MB) 32 us, one of 9000 with 4 key heads (18 MB) 20 us.
#include "nm_common.cuh"

namespace {

constexpr int PAGED_WARPS = 8, PAGED_THREADS = PAGED_WARPS * 32, PAGED_RING = 8192;   // bytes of a warp's ring

// A unit that begins in a block and goes on (nh = 0: none): its last block, row of the output and query heads, and whether it begins where the
// block does (paged_place).
struct PagedJoin {
    int c1, row, h0, nh, first_place;
};

struct PagedArgs {
    nm_attn_paged_desc d;
    const NmTable *exp_tab, *recip_tab;
    int* status;
    int group, blocks_per_head;   // query heads of a key head; units that they make
    int64_t page_bytes, token_bytes;      // distances of pages and tokens in the caches
    NmDivisor by_page;                    // by page_size
    int span;                     // fused: tokens that a block's shared memory holds; split: tokens that a block has at least
    int lead;                     // split: positions without a token before each unit
    int64_t row;                  // split: scores of one head in the workspace
    float *scores, *maxima;       // split: [B][heads][row]; [B][heads], of units that one block has
    float *part_max, *parts;      // split, two places per block: [HEADS]; [HEADS][d] and [HEADS], unit sums not yet joined
    int* tickets;                 // split: per block, how many blocks have finished the unit that begins in it and goes on
    PagedJoin* joins;             // split, for a third launch (otherwise null): per block, the unit that begins in it and goes on
};

__device__ __forceinline__ float paged_table(const NmTable* t, float x)
{
    const float2 kb = t->kb[nm_pwl_index(x, t->inv_h, t->off, (float)(t->n - 1))];
    return __fmaf_rn(kb.x, x, kb.y);
}

// The reciprocal of a row's sum.  Equal segments over all sums from 1 to a long row's length would be far too wide for short rows; with
// recip_pow2 the table sees the sum's mantissa, in [1, 2), and the power of two is undone exactly.
template <typename Table> __device__ __forceinline__ float paged_recip(const PagedArgs& a, float s, Table table)
{
    const uint32_t bits = __float_as_uint(s);
    if (!a.d.recip_pow2 || bits - 0x00800000u >= 0x7f000000u) return table(s);   // (zero, subnormal, negative and not finite as they are)
    return scalbnf(table(__uint_as_float((bits & 0x007fffffu) | 0x3f800000u)), 127 - (int)(bits >> 23));
}
__device__ __forceinline__ float paged_recip(const PagedArgs& a, float s)
{
    return paged_recip(a, s, [&](float x) { return paged_table(a.recip_tab, x); });
}

// The exponential's table in shared memory.  floor(u) is taken by adding 1.5 * 2^23 with rounding down, which leaves it in the low bits
// (0 <= u < 2^22), and the entry's address is formed from those.
struct PagedExp {
    uint32_t at;   // shared address of the table, less what the bits of 1.5 * 2^23 add to it
    float inv_h, off, nm1;
    __device__ __forceinline__ float operator()(float x) const
    {
        const float u = fminf(fmaxf(__fmaf_rn(x, inv_h, off), 0.0f), nm1);
        const uint32_t entry = (__float_as_uint(__fadd_rd(u, 12582912.0f)) << 3) + at;
        float k, b;
        asm("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(k), "=f"(b) : "r"(entry));   // the table is only read
        return __fmaf_rn(k, x, b);
    }
};

// The length of request b and the row of its query and output; row -1 where nothing is read or written for it: it has no new token, or its
// length or row is outside what the call was made for (*error).
struct PagedRequest {
    int len, row;
};
__device__ __forceinline__ PagedRequest paged_request(const PagedArgs& a, int b, int* error)
{
    const int n = a.d.lengths[b];
    int row = b;
    bool good = true;
    if (a.d.token_start) {
        const int start = a.d.token_start[b], end = a.d.token_start[b + 1];
        good = start >= 0 && end >= start && end <= a.d.rows;
        row = end > start ? end - 1 : -1;
    }
    *error = !good ? (int)NM_ERR_INVALID_ARG : row >= 0 && (n < 0 || n > a.d.max_len) ? (int)NM_ERR_SHAPE : 0;
    return *error || row < 0 ? PagedRequest{0, -1} : PagedRequest{n, row};
}

// The tokens of one unit that a block works on.
struct PagedTokens {
    const int32_t* table;   // the request's
    int first, count;
};

// Where a warp's next tiles are: byte offsets from the key head's first token in K and V.  Tokens of a page that the cache does not have
// (recorded) and those that fill up the last tile are PAGED_NONE, read as zeros.  The lanes look up a round of 32 tokens at a time
// (32 / TILE tiles of the warp); the next round's pages are on their way meanwhile.
constexpr int64_t PAGED_NONE = -1;
template <int TILE> struct PagedCursor {
    static constexpr int TILES = 32 / TILE, STEP = 32 * PAGED_WARPS;   // tokens of the block's warps in a round
    const PagedArgs& a;
    const PagedTokens& tok;
    int64_t* buf;   // two rounds, the warp's own
    int token, page, place;   // the lane's token of the next round; its page and place
    uint32_t live;  // lanes of the current round with a token to read

    __device__ __forceinline__ PagedCursor(const PagedArgs& args, const PagedTokens& t, int64_t* b) : a(args), tok(t), buf(b), live(0)
    {
        const int lane = threadIdx.x & 31;
        token = (threadIdx.x >> 5) * TILE + lane / TILE * (PAGED_WARPS * TILE) + lane % TILE;
        look();
    }
    __device__ __forceinline__ void look()
    {
        const int j = tok.first + token, entry = a.by_page(j);
        place = j - entry * a.d.page_size;
        page = token < tok.count ? tok.table[entry] : -1;
    }
    // offsets of the warp's tile number n (one after another from 0); *whole: all of its tokens are there
    __device__ __forceinline__ const int64_t* tile(int n, bool* whole)
    {
        int64_t* at = buf + (n / TILES & 1) * 32;
        if (n % TILES == 0) {
            const bool good = (uint32_t)page < (uint32_t)a.d.num_pages;
            if (!good && token < tok.count) atomicExch(a.status, (int)NM_ERR_INVALID_ARG);
            at[threadIdx.x & 31] = good ? (int64_t)page * a.page_bytes + (int64_t)place * a.token_bytes : PAGED_NONE;
            live = __ballot_sync(0xffffffffu, good);   // (and the lanes' offsets are there)
            __syncwarp();
            token += STEP;
            look();
        }
        constexpr uint32_t ALL = TILE == 32 ? 0xffffffffu : (1u << (TILE & 31)) - 1;
        *whole = (live >> (n % TILES * TILE) & ALL) == ALL;
        return at + n % TILES * TILE;
    }
};

// Asynchronous copies of 16 bytes of a token: a warp copies what it will read itself, so its tiles need no barrier of the block.
__device__ __forceinline__ void paged_copy(uint32_t dst, const uint8_t* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void paged_copy_or_zero(uint32_t dst, const uint8_t* base, int64_t off)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(off < 0 ? base : base + off), "r"(off < 0 ? 0 : 16) : "memory");
}
__device__ __forceinline__ void paged_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void paged_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Runs a warp's tiles through its ring: fetch(n, stage) starts the copies of its tile number n, take(stage) brings a tile from the ring
// to registers, after which the stage is filled again, use(i0) works on the registers.  So all stages are on their way while a tile is
// worked on.  `ready` is called once the first tiles are on their way.
template <int STAGES, int TILE, typename Fetch, typename Ready, typename Take, typename Use>
__device__ __forceinline__ void paged_pipeline(int count, Fetch fetch, Ready ready, Take take, Use use)
{
    constexpr int STEP = PAGED_WARPS * TILE;
    int i0 = (threadIdx.x >> 5) * TILE, next = i0, n = 0, stage = 0;
#pragma unroll
    for (int s = 0; s < STAGES; ++s, next += STEP) {
        if (next < count) fetch(n++, s);
        paged_commit();
    }
    ready();
    for (; i0 < count; i0 += STEP, next += STEP) {
        paged_wait<STAGES - 1>();
        __syncwarp();   // the lanes' copies are there
        take(stage);
        __syncwarp();   // and have been read
        if (next < count) fetch(n++, stage);
        paged_commit();
        use(i0);
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
// Two probabilities as three packed 16-bit terms each, w[2] the largest; term number t counts LIFT^(t - 2)-fold.  Each term but the last is
// the remainder so far rounded towards zero and, being cut from a value one unit lower, always smaller than the remainder: the next
// one is never zero and has the same sign, so an infinite V gives an infinity and not 0 * inf.
//   bf16   8 bits a term: the three add up to e exactly
//   fp16   11 bits a term, but fp16 ends at 2^-24, where a row of many small probabilities has much of its sum.  So what a term leaves,
//          at most 2^-10 of the power of two below it, is multiplied by 2^10: nothing overflows that did not before, and e is
//          exact from 2^-21 on and to 2^-45 below (an |e| below 2^-24 has no first term: it gives NaN with an infinite V)
template <typename T> struct PagedTerms;
template <> struct PagedTerms<__nv_bfloat16> {
    static constexpr float LIFT = 1.f;
    static __device__ __forceinline__ uint32_t cut(float& a, float& b)
    {
        const uint32_t x = __float_as_uint(__fmul_rz(a, 0x1.fffffep-1f)), y = __float_as_uint(__fmul_rz(b, 0x1.fffffep-1f));
        a -= __uint_as_float(x & 0xffff0000u);
        b -= __uint_as_float(y & 0xffff0000u);
        return __byte_perm(x, y, 0x7632);
    }
    static __device__ __forceinline__ uint32_t last(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); }
};
template <> struct PagedTerms<__half> {
    static constexpr float LIFT = 1024.f;
    static __device__ __forceinline__ uint32_t cut(float& a, float& b)
    {
        uint32_t w;
        asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(__fmul_rz(b, 0x1.fffffep-1f)), "f"(__fmul_rz(a, 0x1.fffffep-1f)));
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w));
        a = (a - h.x) * LIFT;
        b = (b - h.y) * LIFT;
        return w;
    }
    static __device__ __forceinline__ uint32_t last(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

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

// Tiles of MT * 16 tokens, NT tiles of 8 query heads: S^T = K Q^T and O^T = V^T P^T, tokens or channels as rows, so that eight heads fill
// a product.  Rows are copied whole and lie in the ring with their 16-byte pieces permuted, piece c of row r at c ^ (r & 7) (rows of
// 96 channels one piece apart instead): neither the copies nor the matrix reads collide.  Probabilities are three 16-bit terms (PagedTerms).
template <typename T, int D_, int NT> struct PagedMma {
    using Elem = T;
    static constexpr int D = D_, HEADS = NT * 8, MT = D <= 64 ? 2 : 1, TILE = 16 * MT, LANES = D / 8;   // lanes of a row
    static constexpr bool POW2 = (LANES & (LANES - 1)) == 0;
    static constexpr int PITCH = D * 2 + (POW2 ? 0 : 16), STAGE = TILE * PITCH, STAGES = PAGED_RING / STAGE < 2 ? 2 : PAGED_RING / STAGE;
    static constexpr int RING = STAGES * STAGE;   // bytes of a warp
    static_assert(D % 32 == 0 && HEADS * D * 4 <= RING, "whole 32-channel pieces; a warp's sums fit its ring");
    static __device__ __forceinline__ float2 read(const float* s) { return *reinterpret_cast<const float2*>(s); }   // two tokens' scores

    static __device__ __forceinline__ uint32_t piece(int row, int c) { return row * PITCH + ((POW2 ? c ^ (row & 7) : c) << 4); }
    static __device__ __forceinline__ void fetch(const T* base, PagedCursor<TILE>& cursor, uint32_t ring_at, int n, int stage)
    {
        const int lane = threadIdx.x & 31;
        bool whole;
        const int64_t* off = cursor.tile(n, &whole);
        const uint32_t to = ring_at + stage * STAGE;
        if constexpr (POW2) {   // the lane has one place in every row that it copies
            const uint8_t* from = (const uint8_t*)base + lane % LANES * 16;
            constexpr int STEP = 32 / LANES;   // rows of a copy
            if (whole) {
#pragma unroll
                for (int x = 0; x < TILE / STEP; ++x) paged_copy(to + piece(x * STEP + lane / LANES, lane % LANES), from + off[x * STEP + lane / LANES]);
            } else {
#pragma unroll
                for (int x = 0; x < TILE / STEP; ++x)
                    paged_copy_or_zero(to + piece(x * STEP + lane / LANES, lane % LANES), from, off[x * STEP + lane / LANES]);
            }
        } else {
#pragma unroll
            for (int x = 0; x < TILE * LANES / 32; ++x) {
                const int at = x * 32 + lane, row = at / LANES, c = at % LANES;
                paged_copy_or_zero(to + piece(row, c), (const uint8_t*)base + c * 16, off[row]);
            }
        }
    }

    // put(h, i, s) takes the score of head h and token i; the heads' maxima over the warp's tokens go to warp_max
    template <typename Put>
    static __device__ __forceinline__ void scores(const PagedArgs& a, const T* Q, int nh, const T* K, const PagedTokens& tok, unsigned char* ring,
                                                  int64_t* offsets, float* warp_max, Put put)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, count = tok.count;
        const uint32_t ring_at = nm_smem_u32(ring);
        PagedCursor<TILE> cursor(a, tok, offsets);
        uint32_t q[NT][D / 16][2], k[MT][D / 16][4];
        float m[NT][2];
        paged_pipeline<STAGES, TILE>(
            count, [&](int n, int stage) { fetch(K, cursor, ring_at, n, stage); },
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
            [&](int stage) {
#pragma unroll
                for (int x = 0; x < MT; ++x)
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) paged_ldmatrix(k[x][c], ring_at + stage * STAGE + piece(x * 16 + (lane & 15), 2 * c + (lane >> 4)));
            },
            [&](int i0) {
                float s[MT][NT][4], s2[MT][NT][4];   // two chains: a product waits for the one before it
#pragma unroll
                for (int x = 0; x < MT; ++x)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[x][n][r] = s2[x][n][r] = 0.f;
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
#pragma unroll
                    for (int x = 0; x < MT; ++x)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            paged_mma(c & 1 ? s2[x][n] : s[x][n], k[x][c][0], k[x][c][1], k[x][c][2], k[x][c][3], q[n][c][0], q[n][c][1], T());
                const bool whole = i0 + TILE <= count;
#pragma unroll
                for (int x = 0; x < MT; ++x)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float v = (s[x][n][r] + s2[x][n][r]) * a.d.scale;
                            const int j = i0 + x * 16 + g + (r >> 1) * 8;
                            if (whole || j < count) {
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
    static __device__ __forceinline__ void values(const PagedArgs& a, int nh, const T* V, const PagedTokens& tok, PagedExp exp, unsigned char* ring,
                                                  int64_t* offsets, float* warp_sum, Max maxima, Get get)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, count = tok.count;
        const uint32_t ring_at = nm_smem_u32(ring);
        PagedCursor<TILE> cursor(a, tok, offsets);
        uint32_t v[MT][D / 16][4];   // channels c * 16 + 0..7 and 8..15 of tokens 0..7, then of tokens 8..15
        float acc[NT][D / 16][4], sum[NT], m[NT];
        float2 next[MT][NT][2];   // scores of the next tile
        // (heads behind the last one read its scores: their sums are dropped)
        auto look = [&](int n, int i0) {
#pragma unroll
            for (int x = 0; x < MT; ++x)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int i = i0 + x * 16 + 2 * t + r * 8;   // a row's storage has whole 32s
                    if (i < count) next[x][n][r] = get(min(n * 8 + g, nh - 1), i);
                }
        };
        paged_pipeline<STAGES, TILE>(
            count, [&](int n, int stage) { fetch(V, cursor, ring_at, n, stage); },
            [&] {
                const float* x = maxima();
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    m[n] = x[min(n * 8 + g, nh - 1)];
                    sum[n] = 0.f;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) acc[n][c][0] = acc[n][c][1] = acc[n][c][2] = acc[n][c][3] = 0.f;
                }
#pragma unroll
                for (int y = 0; y < MT * NT * 2; ++y) next[y / (NT * 2)][y / 2 % NT][y & 1] = make_float2(0.f, 0.f);
#pragma unroll
                for (int n = 0; n < NT; ++n) look(n, (threadIdx.x >> 5) * TILE);
            },
            [&](int stage) {
#pragma unroll
                for (int x = 0; x < MT; ++x)
#pragma unroll
                    for (int c = 0; c < D / 16; ++c)
                        paged_ldmatrix_trans(v[x][c], ring_at + stage * STAGE + piece(x * 16 + (lane & 7) + (lane >> 4) * 8, 2 * c + ((lane >> 3) & 1)));
            },
            [&](int i0) {
                const bool whole = i0 + TILE <= count;
                using Terms = PagedTerms<T>;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint32_t w[3][MT][2];
#pragma unroll
                    for (int x = 0; x < MT; ++x)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float p0 = exp(next[x][n][r].x - m[n]), p1 = exp(next[x][n][r].y - m[n]);
                            if (!whole) {
                                const int i = i0 + x * 16 + 2 * t + r * 8;
                                p0 = i < count ? p0 : 0.f;
                                p1 = i + 1 < count ? p1 : 0.f;
                            }
                            sum[n] += p0 + p1;
                            w[2][x][r] = Terms::cut(p0, p1);
                            w[1][x][r] = Terms::cut(p0, p1);
                            w[0][x][r] = Terms::last(p0, p1);
                        }
                    look(n, i0 + PAGED_WARPS * TILE);
                    // The tensor core truncates its sums: a tile's products have a sum of their own, smallest terms first, and are added
                    // to those of the tiles before in fp32, rounded to nearest.  A product waits for the one before it, so with registers to
                    // spare SIDE channel pieces go side by side, and the 16s of tokens apart (one row of 131071 tokens, fp16, 128 channels: 102 us
                    // with four pieces, 111 with one; 64 requests of up to 4096 tokens, bf16, 64 channels: 66.2 us with the tokens apart, 67.6).
                    constexpr int SIDE = NT > 1 ? 1 : D % 64 == 0 ? 4 : 3, APART = NT > 1 ? 1 : MT, SUMS = SIDE * APART;
#pragma unroll
                    for (int c0 = 0; c0 < D / 16; c0 += SIDE) {
                        float o[SUMS][4];
#pragma unroll
                        for (int c = 0; c < SUMS; ++c) o[c][0] = o[c][1] = o[c][2] = o[c][3] = 0.f;
#pragma unroll
                        for (int y = 0; y < 3; ++y) {
#pragma unroll
                            for (int x = 0; x < MT; ++x)
#pragma unroll
                                for (int c = 0; c < SIDE; ++c)
                                    paged_mma(o[x % APART * SIDE + c], v[x][c0 + c][0], v[x][c0 + c][1], v[x][c0 + c][2], v[x][c0 + c][3], w[y][x][0], w[y][x][1],
                                              T());
                            if (Terms::LIFT != 1.f && y < 2) {
#pragma unroll
                                for (int c = 0; c < SUMS; ++c)
#pragma unroll
                                    for (int r = 0; r < 4; ++r) o[c][r] *= 1.f / Terms::LIFT;
                            }
                        }
#pragma unroll
                        for (int c = 0; c < SIDE; ++c)
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[n][c0 + c][r] += APART == 1 ? o[c][r] : o[c][r] + o[SUMS - SIDE + c][r];
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

    static __device__ __forceinline__ void fetch(const PagedArgs& a, const T* base, PagedCursor<TILE>& cursor, uint32_t ring_at, int n, int stage)
    {
        const int lane = threadIdx.x & 31, part = lane & (LPK - 1), sub = lane / LPK;
        bool whole;
        const int64_t* off = cursor.tile(n, &whole);
        const uint32_t to = ring_at + stage * STAGE + lane * 16;
        const uint8_t* from = (const uint8_t*)(base + part * N);
        if (whole && a.d.d == D) {
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int v = 0; v < VPL; ++v) paged_copy(to + (k * VPL + v) * 512, from + off[k * SUB + sub] + v * (LPK * 16));
        } else {
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int v = 0; v < VPL; ++v) {
                    const bool has = (v * LPK + part) * N < a.d.d;
                    paged_copy_or_zero(to + (k * VPL + v) * 512, has ? from + v * (LPK * 16) : (const uint8_t*)base, has ? off[k * SUB + sub] : PAGED_NONE);
                }
        }
    }
    static __device__ __forceinline__ void take(Vec16<T> (&x)[U][VPL], const unsigned char* ring, int stage)
    {
        const uint4* tile = reinterpret_cast<const uint4*>(ring + stage * STAGE) + (threadIdx.x & 31);
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int v = 0; v < VPL; ++v) x[k][v].raw = tile[(k * VPL + v) * 32];
    }

    template <typename Put>
    static __device__ __forceinline__ void scores(const PagedArgs& a, const T* Q, int nh, const T* K, const PagedTokens& tok, unsigned char* ring, int64_t* offsets,
                                                  float* warp_max, Put put)
    {
        using Sums = PagedSums<HB * U, LPK>;   // sum number k * HB + h: token k, head h
        const int lane = threadIdx.x & 31, part = lane & (LPK - 1), sub = lane / LPK;
        const int count = tok.count;
        const uint32_t ring_at = nm_smem_u32(ring);
        PagedCursor<TILE> cursor(a, tok, offsets);
        const int sum0 = Sums::first(part);
        Vec16<T> x[U][VPL];
        float q[HB][VPL][N], m[Sums::LEFT];
        paged_pipeline<STAGES, TILE>(
            count, [&](int n, int stage) { fetch(a, K, cursor, ring_at, n, stage); },
            [&] {
#pragma unroll
                for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        const int c = (v * LPK + part) * N;
                        Vec16<T> y;
                        y.raw = h < nh && c < a.d.d ? *reinterpret_cast<const uint4*>(Q + h * a.d.d + c) : make_uint4(0, 0, 0, 0);
                        y.get(q[h][v]);
                    }
#pragma unroll
                for (int i = 0; i < Sums::LEFT; ++i) m[i] = -INFINITY;
            },
            [&](int stage) { take(x, ring, stage); },
            [&](int i0) {
                float dot[HB * U];
#pragma unroll
                for (int k = 0; k < U; ++k) {
#pragma unroll
                    for (int h = 0; h < HB; ++h) dot[k * HB + h] = 0.f;
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        float f[N];
                        x[k][v].get(f);
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
    static __device__ __forceinline__ void values(const PagedArgs& a, int nh, const T* V, const PagedTokens& tok, PagedExp exp, unsigned char* ring, int64_t* offsets,
                                                  float* warp_sum, Max maxima, Get get)
    {
        const int lane = threadIdx.x & 31, part = lane & (LPK - 1), sub = lane / LPK;
        const int count = tok.count;
        const uint32_t ring_at = nm_smem_u32(ring);
        PagedCursor<TILE> cursor(a, tok, offsets);
        constexpr int TH = U * HB;   // a token's exponentials are shared by its lanes: lane `part` computes number part, part + LPK, ...
        constexpr int MINE = (TH + LPK - 1) / LPK;
        Vec16<T> x[U][VPL];
        float acc[HB][VPL][N], sum[MINE], m[MINE], next[MINE];   // next: scores of the next tile
        auto look = [&](int i0) {
#pragma unroll
            for (int l = 0; l < MINE; ++l) {
                const int y = l * LPK + part, h = y % HB, i = i0 + y / HB * SUB + sub;
                next[l] = y < TH && h < nh && i < count ? get(h, i) : 0.f;
            }
        };
        paged_pipeline<STAGES, TILE>(
            count, [&](int n, int stage) { fetch(a, V, cursor, ring_at, n, stage); },
            [&] {
                const float* max = maxima();
#pragma unroll
                for (int l = 0; l < MINE; ++l) {
                    m[l] = max[(l * LPK + part) % HB];
                    sum[l] = 0.f;
                }
#pragma unroll
                for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int v = 0; v < VPL; ++v)
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[h][v][e] = 0.f;
                look((threadIdx.x >> 5) * TILE);
            },
            [&](int stage) { take(x, ring, stage); },
            [&](int i0) {
                float mine[MINE];
#pragma unroll
                for (int l = 0; l < MINE; ++l) {
                    const int y = l * LPK + part, h = y % HB, i = i0 + y / HB * SUB + sub;
                    mine[l] = y < TH && h < nh && i < count ? exp(next[l] - m[l]) : 0.f;
                    sum[l] += mine[l];
                }
                look(i0 + PAGED_WARPS * TILE);
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    float e[HB];
#pragma unroll
                    for (int h = 0; h < HB; ++h)
                        e[h] = __shfl_sync(0xffffffffu, mine[(k * HB + h) / LPK], (lane & ~(LPK - 1)) | ((k * HB + h) % LPK));
#pragma unroll
                    for (int v = 0; v < VPL; ++v) {
                        float f[N];
                        x[k][v].get(f);
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
// blocks of an SM: rings of 64 KB leave room for two
constexpr int paged_blocks(int ring) { return ring > 8192 ? 1 : 2; }
constexpr size_t PAGED_OFFSETS = PAGED_WARPS * 64 * 8;   // the cursors' rounds
template <class Core> constexpr size_t paged_split_bytes() { return (size_t)PAGED_WARPS * Core::RING + PAGED_OFFSETS; }
template <class Core> constexpr size_t paged_fused_bytes(int span) { return paged_split_bytes<Core>() + (size_t)Core::HEADS * paged_pitch(span) * 4; }

#define NM_PAGED_EXP_TABLE()                                                                             \
    __shared__ float2 s_exp[NM_MAX_SEGMENTS];                                                            \
    for (int i = threadIdx.x; i < a.exp_tab->n; i += PAGED_THREADS) s_exp[i] = a.exp_tab->kb[i];         \
    const PagedExp exp = {nm_smem_u32(s_exp) - (0x4B400000u << 3), a.exp_tab->inv_h, a.exp_tab->off, (float)(a.exp_tab->n - 1)}

// One launch: a cluster per unit, its blocks sharing the row's tokens evenly.
template <class Core>
__global__ void __launch_bounds__(PAGED_THREADS, paged_blocks(Core::RING)) paged_fused_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    extern __shared__ __align__(128) unsigned char paged_smem[];
    __shared__ float s_max[PAGED_WARPS][Core::HEADS], s_block_max[Core::HEADS], s_row_max[Core::HEADS];
    __shared__ float s_sum[PAGED_WARPS][Core::HEADS], s_block_sum[Core::HEADS];
    NM_PAGED_EXP_TABLE();
    uint32_t ctas;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const int rank = (int)nm_cluster_ctarank();
    const PagedUnit u = paged_unit<Core>(a, blockIdx.x / ctas);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    int error;
    const PagedRequest request = paged_request(a, u.b, &error);
    if (error && threadIdx.x == 0) atomicExch(a.status, error);
    if (request.row < 0) return;   // the whole cluster
    const int len = request.len;
    const int per = ((len + (int)ctas - 1) / (int)ctas + 31) / 32 * 32, first = min(len, rank * per);
    const PagedTokens tok = {a.d.block_tables + (int64_t)u.b * a.d.ld_tables, first, min(len - first, per)};
    const int pitch = paged_pitch(a.span), warp = threadIdx.x >> 5;
    unsigned char* ring = paged_smem + warp * Core::RING;
    int64_t* offsets = reinterpret_cast<int64_t*>(paged_smem + PAGED_WARPS * Core::RING) + warp * 64;
    float* sc = reinterpret_cast<float*>(paged_smem + PAGED_WARPS * Core::RING + PAGED_OFFSETS);
    Core::scores(a, (const T*)a.d.Q + (int64_t)request.row * a.d.ld_q + (int64_t)u.h0 * a.d.d, u.nh, (const T*)a.d.k_cache + (int64_t)u.kv * a.d.stride_head,
                 tok, ring, offsets, s_max[warp], [&](int h, int i, float s) { sc[h * pitch + i] = s; });
    Core::values(
        a, u.nh, (const T*)a.d.v_cache + (int64_t)u.kv * a.d.stride_head, tok, exp, ring, offsets, s_sum[warp],
        [&] {   // the row's maxima
            __syncthreads();
            if (threadIdx.x < Core::HEADS) {
                float x = s_max[0][threadIdx.x];
                for (int w = 1; w < PAGED_WARPS; ++w) x = fmaxf(x, s_max[w][threadIdx.x]);
                s_block_max[threadIdx.x] = x;
                if (ctas == 1) s_row_max[threadIdx.x] = x;
            }
            if (ctas > 1) {   // the other blocks' maxima are read once all of them have come this far
                nm_cluster_sync();
                if (threadIdx.x < Core::HEADS) {
                    float x = -INFINITY;
                    for (uint32_t r = 0; r < ctas; ++r) {
                        float y;
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y) : "r"(nm_mapa(nm_smem_u32(&s_block_max[threadIdx.x]), r)) : "memory");
                        x = fmaxf(x, y);
                    }
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
        ((T*)a.d.out)[(int64_t)request.row * a.d.ld_out + (int64_t)(u.h0 + h) * a.d.d + c] = NmType<T>::from_f(len ? o * paged_recip(a, s) : 0.f);
    }
    if (ctas > 1) nm_cluster_sync();   // no block leaves while another reads its shared memory
}

// Split form.  All requests' units lie one after another (paged_width); block i has positions [i * share, (i + 1) * share).
// Its part of one unit is a segment.  A unit that lies in several blocks has one segment in each: the block's head segment where the
// unit covers the block's first position, its tail segment otherwise, so a block has room for the sums of two.
struct PagedShare {
    int64_t share, pos, end, row0;   // the block's positions still to do; where the current request's first unit begins
    int b, len, row;                 // the current request
};
__device__ __forceinline__ int paged_len32(int len) { return (len + 31) & ~31; }

// Positions of a unit: some without a token, for what a segment costs next to its tokens, then its tokens as whole 32s.
__device__ __forceinline__ int64_t paged_width(const PagedArgs& a, int len) { return len ? (int64_t)a.lead + paged_len32(len) : 0; }

// Length of request b for the shares: 0 where nothing is done for it.
__device__ __forceinline__ int paged_length_or_0(const PagedArgs& a, int b)
{
    int error;
    return paged_request(a, b, &error).len;
}
__device__ __forceinline__ void paged_go_to(const PagedArgs& a, PagedShare& s, int b)
{
    int error;
    const PagedRequest r = paged_request(a, b, &error);
    s.b = b;
    s.len = r.len;
    s.row = r.row;
}

// The block's share: two passes over the lengths, 256 requests at a time.
__device__ __forceinline__ PagedShare paged_share(const PagedArgs& a, int units)
{
    __shared__ int64_t s_warp[PAGED_WARPS], s_row0;
    __shared__ int s_b;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int64_t mine = 0;
    for (int b = tid; b < a.d.B; b += PAGED_THREADS) mine += paged_width(a, paged_length_or_0(a, b));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) s_warp[warp] = mine;
    if (tid == 0) s_b = -1;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < PAGED_WARPS; ++w) total += s_warp[w];
    total *= units;
    PagedShare s;
    s.share = ((total + gridDim.x - 1) / gridDim.x + 31) / 32 * 32;
    if (s.share < a.span) s.share = a.span;
    s.pos = (int64_t)blockIdx.x * s.share;
    s.end = s.pos + s.share < total ? s.pos + s.share : total;
    s.b = s.len = s.row = 0;
    s.row0 = 0;
    if (s.pos >= s.end) return s;
    int64_t before = 0;   // of the requests of earlier turns
    for (int b0 = 0; b0 < a.d.B; b0 += PAGED_THREADS) {
        const int b = b0 + tid;
        const int64_t own = b < a.d.B ? paged_width(a, paged_length_or_0(a, b)) * units : 0;
        int64_t x = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) s_warp[warp] = x;
        __syncthreads();
        int64_t at = before;
        for (int w = 0; w < PAGED_WARPS; ++w) {
            if (w < warp) at += s_warp[w];
            before += s_warp[w];
        }
        at += x - own;
        if (at <= s.pos && s.pos < at + own) {   // one thread at most
            s_b = b;
            s_row0 = at;
        }
        if (before > s.pos) break;
    }
    __syncthreads();
    s.row0 = s_row0;
    paged_go_to(a, s, s_b);
    return s;
}
struct PagedSegment {
    int b, row, unit, first, count;   // request, its row, unit of it, tokens
    int64_t from;                // the unit's first position
    bool whole;                  // the unit lies in this block alone
};
// The next segment of the block; false when there is none.
__device__ __forceinline__ bool paged_next(const PagedArgs& a, PagedShare& s, int units, PagedSegment* g)
{
    if (s.pos >= s.end) return false;
    int64_t width = paged_width(a, s.len);
    while (s.pos >= s.row0 + width * units) {   // the next request that has tokens
        s.row0 += width * units;
        paged_go_to(a, s, s.b + 1);
        width = paged_width(a, s.len);
    }
    const int len32 = paged_len32(s.len);
    g->b = s.b;
    g->row = s.row;
    g->unit = (int)((s.pos - s.row0) / width);
    g->from = s.row0 + g->unit * width + a.lead;
    if (s.pos < g->from) s.pos = g->from;
    if (s.pos >= s.end) return false;   // only positions without a token were left
    g->first = (int)(s.pos - g->from);
    const int64_t stop = g->from + len32 < s.end ? g->from + len32 : s.end;
    g->count = min(s.len, (int)(stop - g->from)) - g->first;
    g->whole = g->first == 0 && stop == g->from + len32;
    s.pos = stop;
    return true;
}
// place of block c's sums of the unit that begins at `from`
__device__ __forceinline__ int64_t paged_place(int64_t from, int64_t share, int64_t c) { return 2 * c + (from <= c * share ? 0 : 1); }

template <class Core>
__global__ void __launch_bounds__(PAGED_THREADS, paged_blocks(Core::RING)) paged_scores_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    extern __shared__ __align__(128) unsigned char paged_smem[];
    __shared__ float s_max[PAGED_WARPS][Core::HEADS];
    const int units = a.d.kv_heads * a.blocks_per_head, warp = threadIdx.x >> 5;
    unsigned char* ring = paged_smem + warp * Core::RING;
    int64_t* offsets = reinterpret_cast<int64_t*>(paged_smem + PAGED_WARPS * Core::RING) + warp * 64;
    nm_grid_dependency_wait();
    nm_grid_launch_dependents();   // what came before this launch is complete for the next one too
    if (threadIdx.x == 0) {
        a.tickets[blockIdx.x] = 0;
        if (a.joins) a.joins[blockIdx.x].nh = 0;
    }
    PagedShare share = paged_share(a, units);
    PagedSegment g;
    while (paged_next(a, share, units, &g)) {
        const PagedUnit u = paged_unit<Core>(a, (int64_t)g.b * units + g.unit);
        const PagedTokens tok = {a.d.block_tables + (int64_t)u.b * a.d.ld_tables, g.first, g.count};
        float* sc = a.scores + ((int64_t)u.b * a.d.heads + u.h0) * a.row + g.first;
        Core::scores(a, (const T*)a.d.Q + (int64_t)g.row * a.d.ld_q + (int64_t)u.h0 * a.d.d, u.nh, (const T*)a.d.k_cache + (int64_t)u.kv * a.d.stride_head,
                     tok, ring, offsets, s_max[warp], [&](int h, int i, float s) {
                         if (h < u.nh) sc[h * a.row + i] = s;
                     });
        __syncthreads();
        if ((int)threadIdx.x < u.nh) {
            float x = s_max[0][threadIdx.x];
            for (int w = 1; w < PAGED_WARPS; ++w) x = fmaxf(x, s_max[w][threadIdx.x]);
            if (g.whole) a.maxima[(int64_t)u.b * a.d.heads + u.h0 + threadIdx.x] = x;
            else a.part_max[paged_place(g.from, share.share, blockIdx.x) * Core::HEADS + threadIdx.x] = x;
        }
        __syncthreads();
    }
}

__host__ __device__ constexpr int paged_part_floats(int heads, int d) { return heads * d + (heads + 3) / 4 * 4; }   // [head][channel], then the row sums

// The result of a unit that blocks c0..c1 have: groups of threads take every so manieth block, four channels a thread, eight blocks'
// loads in flight; then the groups' sums are added.  (One thread after another through the blocks, each load waiting for the
// last: 25 us for the 37 blocks of a unit.)
template <class Core, typename T>
__device__ __forceinline__ void paged_join(const PagedArgs& a, int nh, int64_t from, int64_t share, int64_t c0, int64_t c1, float* smem, T* result)
{
    const int d4 = a.d.d / 4, items = nh * d4, groups = items < PAGED_THREADS ? PAGED_THREADS / items : 1, n = (int)(c1 - c0) + 1;
    const int stride = paged_part_floats(Core::HEADS, a.d.d);
    float4* s_out = reinterpret_cast<float4*>(smem);                       // [group][item]
    float* s_sum = smem + groups * items * 4;                              // [group][item]
    for (int y = threadIdx.x; y < groups * items; y += PAGED_THREADS) {
        const int x = y % items, h = x / d4;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        float s = 0.f;
#pragma unroll 8
        for (int i = y / items; i < n; i += groups) {
            const float* p = a.parts + paged_place(from, share, c0 + i) * stride;
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p) + x);
            o.x += v.x;
            o.y += v.y;
            o.z += v.z;
            o.w += v.w;
            s += __ldcg(p + Core::HEADS * a.d.d + h);
        }
        s_out[y] = o;
        s_sum[y] = s;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < items; x += PAGED_THREADS) {
        float4 o = s_out[x];
        float s = s_sum[x];
        for (int g = 1; g < groups; ++g) {
            const float4 v = s_out[g * items + x];
            o.x += v.x;
            o.y += v.y;
            o.z += v.z;
            o.w += v.w;
            s += s_sum[g * items + x];
        }
        const float r = paged_recip(a, s);
        result[x * 4] = NmType<T>::from_f(o.x * r);
        result[x * 4 + 1] = NmType<T>::from_f(o.y * r);
        result[x * 4 + 2] = NmType<T>::from_f(o.z * r);
        result[x * 4 + 3] = NmType<T>::from_f(o.w * r);
    }
}

template <class Core>
__global__ void __launch_bounds__(PAGED_THREADS, paged_blocks(Core::RING)) paged_values_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    extern __shared__ __align__(128) unsigned char paged_smem[];
    __shared__ float s_m[Core::HEADS], s_sum[PAGED_WARPS][Core::HEADS];
    __shared__ int s_last;
    NM_PAGED_EXP_TABLE();
    const int units = a.d.kv_heads * a.blocks_per_head, warp = threadIdx.x >> 5;
    unsigned char* ring = paged_smem + warp * Core::RING;
    int64_t* offsets = reinterpret_cast<int64_t*>(paged_smem + PAGED_WARPS * Core::RING) + warp * 64;
    const float* out = reinterpret_cast<const float*>(paged_smem);
    nm_grid_launch_dependents();
    // Only the scores come from the launch before, which has let this one start once everything before it was complete: lengths, rows,
    // tables and the first values are read before it is done.
    PagedShare share = paged_share(a, units);
    bool waited = false;
    for (int b = blockIdx.x; b < a.d.B; b += gridDim.x) {
        int error;
        const PagedRequest r = paged_request(a, b, &error);
        if (error && threadIdx.x == 0) atomicExch(a.status, error);
        if (r.row >= 0 && r.len == 0) {
            if (!waited) nm_grid_dependency_wait();   // nothing is written before
            waited = true;
            for (int x = threadIdx.x; x < a.d.heads * a.d.d; x += PAGED_THREADS) ((T*)a.d.out)[(int64_t)r.row * a.d.ld_out + x] = NmType<T>::from_f(0.f);
        }
    }
    PagedSegment g;
    while (paged_next(a, share, units, &g)) {
        const PagedUnit u = paged_unit<Core>(a, (int64_t)g.b * units + g.unit);
        const PagedTokens tok = {a.d.block_tables + (int64_t)u.b * a.d.ld_tables, g.first, g.count};
        const int64_t head0 = (int64_t)u.b * a.d.heads + u.h0;
        const int64_t c0 = g.from / share.share, c1 = (g.from + paged_len32(share.len) - 1) / share.share;   // the unit's blocks
        const float* sc = a.scores + head0 * a.row + g.first;
        Core::values(
            a, u.nh, (const T*)a.d.v_cache + (int64_t)u.kv * a.d.stride_head, tok, exp, ring, offsets, s_sum[warp],
            [&] {
                if (!waited) nm_grid_dependency_wait();
                waited = true;
                if (g.whole) {
                    if ((int)threadIdx.x < Core::HEADS) s_m[threadIdx.x] = (int)threadIdx.x < u.nh ? a.maxima[head0 + threadIdx.x] : 0.f;
                } else {
                    const int lane = threadIdx.x & 31;
                    for (int h = warp; h < Core::HEADS; h += PAGED_WARPS) {
                        float m = -INFINITY;
                        if (h < u.nh)
                            for (int64_t c = c0 + lane; c <= c1; c += 32) m = fmaxf(m, a.part_max[paged_place(g.from, share.share, c) * Core::HEADS + h]);
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                        if (lane == 0) s_m[h] = m;
                    }
                }
                __syncthreads();
                return (const float*)s_m;
            },
            [&](int h, int i) { return Core::read(sc + h * a.row + i); });
        __syncthreads();
        T* result = (T*)a.d.out + (int64_t)g.row * a.d.ld_out + (int64_t)u.h0 * a.d.d;
        float* part = a.parts + paged_place(g.from, share.share, blockIdx.x) * paged_part_floats(Core::HEADS, a.d.d);
        for (int x = threadIdx.x; x < u.nh * Core::D; x += PAGED_THREADS) {
            const int h = x / Core::D, c = x - h * Core::D;
            if (c >= a.d.d) continue;
            float o = out[x], s = s_sum[0][h];
            for (int w = 1; w < PAGED_WARPS; ++w) {
                o += out[w * (Core::RING / 4) + x];
                s += s_sum[w][h];
            }
            if (g.whole) {
                result[h * a.d.d + c] = NmType<T>::from_f(o * paged_recip(a, s));
            } else {
                part[h * a.d.d + c] = o;
                if (c == 0) part[Core::HEADS * a.d.d + h] = s;
            }
        }
        if (!g.whole) {   // the unit's last block adds up what all of them left, in their order
            if (a.joins) {
                if (g.first == 0 && threadIdx.x == 0) a.joins[c0] = PagedJoin{(int)c1, g.row, u.h0, u.nh, g.from == c0 * share.share};
                __syncthreads();   // the ring and the sums have been read
                continue;
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                __threadfence();
                s_last = atomicAdd(a.tickets + c0, 1) == (int)(c1 - c0);
                __threadfence();
            }
            __syncthreads();
            if (s_last) paged_join<Core>(a, u.nh, g.from, share.share, c0, c1, reinterpret_cast<float*>(paged_smem), result);
        }
        __syncthreads();   // the ring and the sums have been read
    }
    if (!waited) nm_grid_dependency_wait();   // a launch is not complete before the one it followed
}

// Joins the units that begin in a block and go on: a block per such unit's query head.  Groups of threads take every so manieth of the
// unit's blocks, four channels a thread, eight loads in flight each; then the groups' sums are added.
constexpr int JOIN_THREADS = 512;
template <class Core>
__global__ void __launch_bounds__(JOIN_THREADS) paged_join_kernel(const PagedArgs a)
{
    using T = typename Core::Elem;
    __shared__ float4 s_out[JOIN_THREADS];
    __shared__ float s_sum[JOIN_THREADS];
    __shared__ float2 s_recip[NM_MAX_SEGMENTS];
    const int tid = threadIdx.x, c0 = blockIdx.x / Core::HEADS, h = blockIdx.x % Core::HEADS;
    const float inv_h = a.recip_tab->inv_h, off = a.recip_tab->off, nm1 = (float)(a.recip_tab->n - 1);
    for (int i = tid; i < a.recip_tab->n; i += JOIN_THREADS) s_recip[i] = a.recip_tab->kb[i];
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const PagedJoin j = a.joins[c0];
    if (h >= j.nh) return;
    const int d4 = a.d.d / 4, groups = JOIN_THREADS / d4, n = j.c1 - c0 + 1, x = tid % d4, stride = paged_part_floats(Core::HEADS, a.d.d);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float s = 0.f;
    if (tid < groups * d4) {
        for (int i0 = tid / d4; i0 < n; i0 += 8 * groups) {
            float4 v[8];
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = min(i0 + k * groups, n - 1);
                const float* p = a.parts + (int64_t)(2 * (c0 + i) + (i || j.first_place ? 0 : 1)) * stride;
                v[k] = *reinterpret_cast<const float4*>(p + h * a.d.d + x * 4);
                w[k] = p[Core::HEADS * a.d.d + h];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (i0 + k * groups >= n) break;
                o.x += v[k].x;
                o.y += v[k].y;
                o.z += v[k].z;
                o.w += v[k].w;
                s += w[k];
            }
        }
        s_out[tid] = o;
        s_sum[tid] = s;
    }
    __syncthreads();
    if (tid >= d4) return;
    for (int g = 1; g < groups; ++g) {
        const float4 v = s_out[g * d4 + x];
        o.x += v.x;
        o.y += v.y;
        o.z += v.z;
        o.w += v.w;
        s += s_sum[g * d4 + x];
    }
    const float r = paged_recip(a, s, [&](float x) {
        const float2 kb = s_recip[nm_pwl_index(x, inv_h, off, nm1)];
        return __fmaf_rn(kb.x, x, kb.y);
    });
    T* result = (T*)a.d.out + (int64_t)j.row * a.d.ld_out + (int64_t)(j.h0 + h) * a.d.d + x * 4;
    result[0] = NmType<T>::from_f(o.x * r);
    result[1] = NmType<T>::from_f(o.y * r);
    result[2] = NmType<T>::from_f(o.z * r);
    result[3] = NmType<T>::from_f(o.w * r);
}

// ---------------------------------------------------------------- host

// A segment costs a block some 4 us next to its bytes: the first pages and tokens to arrive, the warps' sums, the join.  So that blocks with
// many short segments do not end last, each unit counts for as many bytes of K more as a block moves meanwhile.  bf16, 8 key heads of 128
// channels, 64 requests of 1 to 4096 tokens: 0 / 32 / 64 / 96 / 128 / 256 KB 145 / 118 / 106 / 104 / 104 / 108 us; 15 requests of 0 to 2898
// tokens 35 / 34 / 33 / 32 / 31 / 32 us; requests of 4096 tokens alike gain nothing.
constexpr int PAGED_LEAD_BYTES = 96 * 1024;
// Units up to which a third launch joins them: each lies in so many blocks that one block takes long to add them up, and waits for the
// last of them first.  bf16, 128 channels, joined in the second launch against a third: 1 unit of 122567 tokens 41 against 32 us, 2 of 50000
// 32 / 28, 4 of 50000 35 / 35, 8 of 65536 60 / 62, 256 of 4096 102 / 110.
constexpr int PAGED_JOIN_UNITS = 4;
constexpr int PAGED_SMS = 148;   // the layout must not depend on the device: the workspace's size is asked for without one

// Query heads of a unit: 16 where the tensor cores take them and the registers hold their sums, otherwise as few as cover the group.
int paged_heads(const nm_attn_paged_desc* d, bool mma)
{
    const int group = d->heads / d->kv_heads;
    if (mma) return group > 8 && d->d <= 128 ? 16 : 8;
    return group >= 8 ? 8 : group >= 4 ? 4 : group >= 2 ? 2 : 1;
}
// Tokens of a block of the fused form: scores take what rings of 64 KB leave of half an SM's shared memory.
int paged_cap(int heads) { return (40 * 1024 - heads * 4 * 40) / (heads * 4) / 32 * 32; }
// Bytes of K and V that a block of a cluster streams at most where the clusters leave SMs idle: split launches use all SMs, and cost some 15 us
// before the first byte.  One request, 4 key heads of 128 channels, fused against split: bf16, 5000 / 9000 tokens 14 / 20 against 18 / 20 us
// (inputs in the L2: 13 / 18); fp32, 5000 / 10000 tokens 25 / 43 against 19 / 23 us, so for fp32 the border lies a little high when the cache is
// cold (inputs in the L2: 21 against 19).
int64_t paged_cluster_bytes(bool mma) { return mma ? 1280 * 1024 : 640 * 1024; }
bool paged_mma_supported(const nm_attn_paged_desc* d) { return d->dtype != NM_F32 && (d->d == 64 || d->d == 96 || d->d == 128 || d->d == 256); }

struct PagedLayout {
    bool mma, fused, join_launch;
    int heads, blocks_per_head, ctas, span;
    int64_t units, row, blocks;
    size_t scores, maxima, part_max, parts, tickets, joins, total;
};
PagedLayout layout_of(const nm_attn_paged_desc* d)
{
    PagedLayout l = PagedLayout();
    const int group = d->heads / d->kv_heads;
    l.mma = paged_mma_supported(d);
    l.heads = paged_heads(d, l.mma);
    l.blocks_per_head = (group + l.heads - 1) / l.heads;
    l.units = (int64_t)d->B * d->kv_heads * l.blocks_per_head;
    const int cap = paged_cap(l.heads);
    int ctas = 1;
    while (ctas < 8 && ((d->max_len + ctas - 1) / ctas > cap || (l.units * ctas * 2 <= 2 * PAGED_SMS && d->max_len > ctas * 128))) ctas *= 2;
    const int64_t block_bytes = (int64_t)((d->max_len + ctas - 1) / ctas) * d->d * 2 * nm_dtype_size(d->dtype);
    l.fused = d->max_len <= ctas * cap && (ctas == 1 || (l.units * ctas <= 2 * PAGED_SMS && (l.units * ctas > PAGED_SMS || block_bytes <= paged_cluster_bytes(l.mma))));
    if (l.fused) {
        l.ctas = ctas;
        l.span = ((d->max_len + ctas - 1) / ctas + 31) / 32 * 32;
        l.blocks = l.units * ctas;
        return l;
    }
    l.ctas = 1;
    l.span = 256;
    l.blocks = PAGED_SMS * (l.mma && d->d == 256 ? 1 : 2);   // one wave
    l.row = ((int64_t)d->max_len + 31) / 32 * 32;
    auto take = [&l](size_t bytes) { const size_t at = l.total; l.total += (bytes + 255) / 256 * 256; return at; };
    l.scores = take((size_t)d->B * d->heads * l.row * 4);
    l.maxima = take((size_t)d->B * d->heads * 4);
    l.part_max = take((size_t)l.blocks * 2 * l.heads * 4);
    l.parts = take((size_t)l.blocks * 2 * paged_part_floats(l.heads, d->d) * 4);
    l.tickets = take((size_t)l.blocks * 4);
    l.join_launch = l.units <= PAGED_JOIN_UNITS;
    if (l.join_launch) l.joins = take((size_t)l.blocks * sizeof(PagedJoin));
    return l;
}

template <typename K>
nm_status paged_launch(nm_ctx* ctx, K kernel, std::atomic<uint64_t>& allowed, const PagedArgs& a, int64_t blocks, int threads, size_t smem, int ctas,
                       double bytes, cudaStream_t st)
{
    if (blocks > INT32_MAX) return NM_ERR_SHAPE;
    // (48 KB are there without asking, the kernels' static arrays among them)
    if (smem > 40 * 1024 && !nm_allow_smem(ctx, (const void*)kernel, 220 * 1024, allowed)) return NM_ERR_CUDA;
    NmLaunchScope scope(ctx, NM_KERNEL_ATTENTION_PAGED, bytes, st);
    NmLaunchConfig lc(ctx, dim3((unsigned)blocks), threads, smem, st, ctas);
    return cudaLaunchKernelEx(&lc.cfg, kernel, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

template <class Core>
nm_status launch(nm_ctx* ctx, const PagedArgs& a, const PagedLayout& l, cudaStream_t st)
{
    using T = typename Core::Elem;
    const double bytes = (double)a.d.B * a.d.max_len * a.d.kv_heads * a.d.d * sizeof(T);
    static std::atomic<uint64_t> allowed[3];
    if (l.fused) return paged_launch(ctx, paged_fused_kernel<Core>, allowed[0], a, l.blocks, PAGED_THREADS, paged_fused_bytes<Core>(l.span), l.ctas, 2 * bytes, st);
    nm_status s = paged_launch(ctx, paged_scores_kernel<Core>, allowed[1], a, l.blocks, PAGED_THREADS, paged_split_bytes<Core>(), 1, bytes, st);
    if (s == NM_OK) s = paged_launch(ctx, paged_values_kernel<Core>, allowed[2], a, l.blocks, PAGED_THREADS, paged_split_bytes<Core>(), 1, bytes, st);
    if (s == NM_OK && l.join_launch) s = paged_launch(ctx, paged_join_kernel<Core>, allowed[0], a, l.blocks * Core::HEADS, JOIN_THREADS, 0, 1, 0.0, st);
    return s;
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
    const int es = (int)nm_dtype_size(d->dtype);
    a.page_bytes = d->stride_page * es;
    a.token_bytes = d->stride_token * es;
    a.by_page = NmDivisor::of(d->page_size);
    a.lead = PAGED_LEAD_BYTES / (d->d * es) / 32 * 32;
    a.row = l.row;
    uint8_t* ws = (uint8_t*)workspace;
    a.scores = (float*)(ws + l.scores);
    a.maxima = (float*)(ws + l.maxima);
    a.part_max = (float*)(ws + l.part_max);
    a.parts = (float*)(ws + l.parts);
    a.tickets = (int*)(ws + l.tickets);
    a.joins = l.join_launch ? (PagedJoin*)(ws + l.joins) : nullptr;
    switch (d->dtype) {
    case NM_F32: return dispatch<float>(ctx, a, l, st);
    case NM_BF16: return dispatch<__nv_bfloat16>(ctx, a, l, st);
    case NM_F16: return dispatch<__half>(ctx, a, l, st);
    default: return NM_ERR_UNSUPPORTED;
    }
}
