// Few tokens times 4-bit weights with group scales, PWL epilogue.
//
// Bound by the weights' bytes as long as the tokens are few.  The weights are the row operand of m16n8k16 products (16 weight rows, 8
// tokens, nothing padded but the last tokens), their codes made 16-bit numbers in registers: a word of eight codes gives pairs
// (k, k + 4) by one mask each, 128 + c (bf16) or 1024 + c (fp16) by the bits, c - 8 by one exact subtraction, so products and their
// sums within a group are those of whole numbers and activations; the group's sum takes its scale in fp32.  tcgen05 would want the
// 16-bit weights written to tensor or shared memory first, four times the bytes that arrive, and the accumulator read back per group; for
// many tokens that would pay (weights are unpacked again for every 32 here), and is not built.
// Measured, bf16, 16384 x 8192 (67 MB of codes: 10.3 us; the copies alone take 14.5 us): 1 token 30 us, 8 tokens 32 us, 32 tokens 52 us,
// 512 tokens 643 us.  Up to 8 tokens the streams are short: 512 blocks on 296 places, four blocks of k a warp for a ring of three stages, so
// rings that fill and drain, sums that are joined and the second wave are most of it.  At 32 tokens fragments from shared memory (2 KB for 256
// bytes of codes), instructions (0.46 per cycle and scheduler, tensor pipe 30 % busy) and 256 blocks on 148 SMs.
// fp32 activations are three bf16 terms (8 + 8 + 8 bits: exact), three products each: 1 / 8 / 16 / 32 tokens 59 / 64 / 118 / 188 us; above 8
// tokens the shared fragments leave one block an SM.
//
// Every warp streams its own weights through a ring of asynchronous copies (256 codes of 16 or 32 rows a stage, so 128 bytes a row):
// no barrier in the loop.  Activations come through L1, shared by the warps of a block that work on the same k.
#include <type_traits>

#include "nm_common.cuh"

namespace {

constexpr int W4_WARPS = 8, W4_THREADS = W4_WARPS * 32, W4_BLOCK_K = 256, W4_TILE = 2048;   // a stage of 16 rows: 128 bytes each
constexpr int W4_MAX_SMEM = 227 * 1024;

struct W4Args {
    nm_linear_w4_desc d;
    const NmTable* tab;
    int row_warps, k_blocks, k_groups, row_blocks;
};

template <typename T> struct W4Type {
    using Mma = T;
    static constexpr int TERMS = 1;
};
template <> struct W4Type<float> {
    using Mma = __nv_bfloat16;
    static constexpr int TERMS = 3;
};

__device__ __forceinline__ void w4_mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void w4_mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1, __half)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The eight codes of a word as pairs (i, i + 4) of whole numbers -8..7.
__device__ __forceinline__ uint32_t w4_sub(uint32_t v, float c, __nv_bfloat16)
{
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), __floats2bfloat162_rn(c, c));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void w4_pairs(uint32_t w, uint32_t* p, __nv_bfloat16)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = w4_sub(((w >> (4 * i)) & 0x000f000fu) | 0x43004300u, 136.f, __nv_bfloat16());   // 128 + c
}
__device__ __forceinline__ void w4_pairs(uint32_t w, uint32_t* p, __half)
{
    // 1024 + c from the low half of a byte, 1024 + 16 c from the high one, which needs no shift: times 1/16, all of it exact
    const uint32_t h = w >> 8, magic = 0x64006400u;
    const uint32_t v[4] = {(w & 0x000f000fu) | magic, (w & 0x00f000f0u) | magic, (h & 0x000f000fu) | magic, (h & 0x00f000f0u) | magic};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 x = *reinterpret_cast<const __half2*>(&v[i]);
        const __half2 r = i & 1 ? __hfma2(x, __floats2half2_rn(0.0625f, 0.0625f), __floats2half2_rn(-72.f, -72.f)) : __hsub2(x, __floats2half2_rn(1032.f, 1032.f));
        p[i] = *reinterpret_cast<const uint32_t*>(&r);
    }
}

// Eight activations of one token as they lie in memory, and as pairs (i, i + 4) for every term.
template <typename T> struct W4Raw {
    static constexpr int VECS = sizeof(T) / 2, TERMS = W4Type<T>::TERMS;
    uint4 v[VECS];
    __device__ __forceinline__ void load(const T* x)
    {
#pragma unroll
        for (int i = 0; i < VECS; ++i) v[i] = __ldg(reinterpret_cast<const uint4*>(x) + i);
    }
    __device__ __forceinline__ void pairs(uint32_t (&p)[TERMS][4]) const
    {
        if constexpr (TERMS == 1) {
            p[0][0] = __byte_perm(v[0].x, v[0].z, 0x5410);
            p[0][1] = __byte_perm(v[0].x, v[0].z, 0x7632);
            p[0][2] = __byte_perm(v[0].y, v[0].w, 0x5410);
            p[0][3] = __byte_perm(v[0].y, v[0].w, 0x7632);
        } else {
            const uint32_t a[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, b[4] = {v[VECS - 1].x, v[VECS - 1].y, v[VECS - 1].z, v[VECS - 1].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t ta[3], tb[3];
                split(a[i], ta);
                split(b[i], tb);
#pragma unroll
                for (int s = 0; s < TERMS; ++s) p[s][i] = __byte_perm(ta[s], tb[s], 0x7632);
            }
        }
    }
    // x as three bf16 numbers in the upper halves: the first two cut off (so none of them overflows), the rest has 8 bits left.
    // What is not finite stays in the first term alone (an infinity's rest would be NaN).
    static __device__ __forceinline__ void split(uint32_t bits, uint32_t* t)
    {
        const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
        t[0] = finite ? bits & 0xffff0000u : (bits & 0x007fffffu) ? 0x7fc00000u : bits;
        const float r = finite ? __uint_as_float(bits) - __uint_as_float(t[0]) : 0.f;
        t[1] = __float_as_uint(r) & 0xffff0000u;
        t[2] = __float_as_uint(r - __uint_as_float(t[1])) & 0xffff0000u;
    }
};

__device__ __forceinline__ void w4_copy(uint32_t dst, const void* src, bool valid)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// NT tiles of 8 tokens, RW tiles of 16 weight rows per warp.  row_warps warps of a block lie along the rows, the others and the
// CTAs of a cluster split k, block by block in turn; their sums are added in that order at the end.
// Activations of up to 8 tokens are loaded by each warp for itself, through L1.  More tokens are shared (STAGED): all warps lay the pairs
// of a slice of k out in shared memory as the products take them, once for all of the block's rows, a slice ahead of their use.
template <typename T, int NT, int RW, int STAGES, int GS>
__global__ void __launch_bounds__(W4_THREADS, 2) linear_w4_kernel(const W4Args a)
{
    using Mma = typename W4Type<T>::Mma;
    constexpr bool STAGED = NT > 1;
    constexpr int TERMS = W4Type<T>::TERMS, RING = STAGES * RW * W4_TILE, PITCH = 16 * RW + 4;
    constexpr int FRAG = NT * TERMS * 512;   // STAGED: pairs of 32 k
    static_assert(NT * 8 * PITCH * 4 <= RING, "a warp's sums fit its ring");
    extern __shared__ __align__(128) unsigned char w4_smem[];
    const nm_linear_w4_desc& d = a.d;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int row_warp = warp % a.row_warps, k_warp = warp / a.row_warps, k_warps = W4_WARPS / a.row_warps;
    uint32_t ctas;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t rank = nm_cluster_ctarank();
    const uint32_t unit = blockIdx.x / ctas;
    const int64_t m0 = (int64_t)(unit / a.row_blocks) * (NT * 8), block_row = (int64_t)(unit % a.row_blocks) * (16 * RW * a.row_warps);
    const int64_t n0 = block_row + row_warp * (16 * RW);
    const int step = k_warps * (int)ctas, first = (int)rank * k_warps + k_warp;
    unsigned char* ring = w4_smem + warp * RING;
    const uint32_t ring_at = nm_smem_u32(ring);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();

    // 16-byte piece c of a row lies at place c ^ (row & 7): word reads hit all banks.  Rows behind the last one are read as its copy, their
    // sums are not stored.
    const int copy_row = lane >> 3, copy_chunk = lane & 7;
    const uint8_t* from[RW * 4];
#pragma unroll
    for (int r = 0; r < RW * 4; ++r)
        from[r] = d.codes + (n0 + r * 4 + copy_row < d.N ? n0 + r * 4 + copy_row : d.N - 1) * d.ld_codes + copy_chunk * 16;
    const uint32_t to[2] = {ring_at + copy_row * 128 + ((copy_chunk ^ copy_row) << 4), ring_at + (copy_row + 4) * 128 + ((copy_chunk ^ (copy_row + 4)) << 4)};
    auto fetch = [&](int b, int stage) {
        if (b < a.k_blocks) {
            const int64_t at = (int64_t)b * (W4_BLOCK_K / 2);
            const bool valid = b + 1 < a.k_blocks || (at + copy_chunk * 16) * 2 < d.K;   // the last block may be short
#pragma unroll
            for (int r = 0; r < RW * 4; ++r)
                w4_copy(to[r & 1] + (r >> 1) * 1024 + stage * (RW * W4_TILE), valid ? from[r] + at : d.codes, valid);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float sum[RW][NT][4];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[r][n][i] = 0.f;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(first + s * step, s);

    constexpr int groups = 8 / GS;   // of a block
    // Scales of groups t and t + 4 of a block, of rows g and g + 8; handed round among four lanes below.  The next block's are on their
    // way while one is worked on: they lie a row apart, and so far apart that each load waits for memory.
    const T* scales[RW][2];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t row = n0 + r * 16 + h * 8 + g;
            scales[r][h] = (const T*)d.scales + (row < d.N ? row : d.N - 1) * d.ld_scales + t;
        }
    T sc[RW][2][2], sc_next[RW][2][2];
    auto look = [&](int b) {
        if (b >= a.k_blocks) return;
        const int at = b * groups, left = a.k_groups - at;   // groups of a row fit 31 bits
#pragma unroll
        for (int q = 0; q < (GS == 1 ? 2 : 1); ++q)
            if (t + 4 * q < groups && t + 4 * q < left) {
#pragma unroll
                for (int r = 0; r < RW; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) sc_next[r][h][q] = scales[r][h][at + 4 * q];
            }
    };
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) sc_next[r][h][0] = sc_next[r][h][1] = NmType<T>::from_f(0.f);
    look(first);
    const T* acts[NT];   // (tokens behind the last one are read as its copy, their sums are not stored)
#pragma unroll
    for (int n = 0; n < NT; ++n) acts[n] = (const T*)d.A + (m0 + n * 8 + g < d.M ? m0 + n * 8 + g : d.M - 1) * d.lda + t * 8;
    // STAGED: warp w lays out step w of each of the slice's k_warps blocks (at most 4 / NT)
    constexpr int SLOTS = STAGED ? 4 / NT : 1;
    W4Raw<T> mine[SLOTS][NT];
    unsigned char* shared_acts = w4_smem + W4_WARPS * RING;
    auto gather = [&](int slice) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int64_t at = ((int64_t)slice * k_warps + k) * W4_BLOCK_K + warp * 32;
                if (k < k_warps) mine[k][n].load(acts[n] + (at < d.K ? at : 0));   // (what lies behind K is not used)
            }
    };
    auto lay_out = [&](int half) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (k < k_warps) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint32_t x[TERMS][4];
                    mine[k][n].pairs(x);
#pragma unroll
                    for (int s = 0; s < TERMS; ++s)
                        reinterpret_cast<uint4*>(shared_acts + ((half * k_warps + k) * 8 + warp) * FRAG + (n * TERMS + s) * 512)[lane] =
                            make_uint4(x[s][0], x[s][1], x[s][2], x[s][3]);
                }
            }
    };
    constexpr int CJ = STAGED ? 1 : 4 / W4Raw<T>::VECS;   // steps of 32 k whose activations are loaded ahead
    const int slices = (a.k_blocks + k_warps - 1) / k_warps;
    if constexpr (STAGED) {
        if ((int)rank < slices) {
            gather(rank);
            lay_out(0);
        }
        __syncthreads();
    }
    int stage = 0, half = 0;
    for (int slice = rank; slice < slices; slice += ctas) {   // the same for all warps
        const int b = slice * k_warps + k_warp;
        if constexpr (STAGED) {
            if (slice + (int)ctas < slices) gather(slice + ctas);
        }
        if (b < a.k_blocks) {
            fetch(b + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int q = 0; q < 2; ++q) sc[r][h][q] = sc_next[r][h][q];
            look(b + step);
            const int64_t k0 = (int64_t)b * W4_BLOCK_K;
            const int steps = d.K - k0 >= W4_BLOCK_K ? 8 : (int)(d.K - k0) / 32;   // K is a multiple of 32
            const unsigned char* tile = ring + stage * (RW * W4_TILE);
            const unsigned char* frags = shared_acts + (half * k_warps + k_warp) * 8 * FRAG;
            // FULL: all eight steps, with no branch between them
            auto block = [&](auto full) {
                constexpr bool FULL = decltype(full)::value;
                W4Raw<T> ahead[2][CJ];
                auto load = [&](int j0, W4Raw<T> (&x)[CJ]) {
                    if constexpr (!STAGED) {
#pragma unroll
                        for (int j = 0; j < CJ; ++j) {
                            x[j].load(acts[0] + (FULL || j0 + j < steps ? k0 + (j0 + j) * 32 : 0));
                        }
                    }
                };
                load(0, ahead[0]);
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
                __syncwarp();
                float part[RW][NT][4];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j % CJ == 0 && j + CJ < 8) load(j + CJ, ahead[(j / CJ + 1) & 1]);
                    if (FULL || j < steps) {   // the same for the whole warp
                        uint32_t x[NT][TERMS][4];
                        if constexpr (STAGED) {
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int s = 0; s < TERMS; ++s) {
                                    const uint4 v = reinterpret_cast<const uint4*>(frags + j * FRAG + (n * TERMS + s) * 512)[lane];
                                    x[n][s][0] = v.x, x[n][s][1] = v.y, x[n][s][2] = v.z, x[n][s][3] = v.w;
                                }
                        } else {
                            ahead[(j / CJ) & 1][j % CJ].pairs(x[0]);
                        }
                        if (j % GS == 0) {
#pragma unroll
                            for (int r = 0; r < RW; ++r)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) part[r][n][i] = 0.f;
                        }
                        auto weights = [&](int r, uint32_t* lo, uint32_t* hi) {
                            const uint32_t w0 = *reinterpret_cast<const uint32_t*>(tile + (r * 16 + g) * 128 + ((j ^ g) << 4) + t * 4);
                            const uint32_t w1 = *reinterpret_cast<const uint32_t*>(tile + (r * 16 + g + 8) * 128 + ((j ^ g) << 4) + t * 4);
                            w4_pairs(w0, lo, Mma());
                            w4_pairs(w1, hi, Mma());
                        };
                        if constexpr (TERMS == 1) {
#pragma unroll
                            for (int r = 0; r < RW; ++r) {
                                uint32_t lo[4], hi[4];
                                weights(r, lo, hi);
#pragma unroll
                                for (int p = 0; p < 4; p += 2) {
                                    const uint32_t f[4] = {lo[p], hi[p], lo[p + 1], hi[p + 1]};
#pragma unroll
                                    for (int n = 0; n < NT; ++n) w4_mma(part[r][n], f, x[n][0][p], x[n][0][p + 1], Mma());
                                }
                            }
                        } else {
                            // The tensor core truncates its sums.  With three terms a group would be a chain of 6 to 24 products, whose
                            // truncations show in fp32 (operands of one sign, K 128: 18 units of 2^-24 too little).  So the 32 k of a step have
                            // a sum of their own, smallest terms first, and are added in fp32: two truncations count, half a unit in all.
                            uint32_t lo[RW][4], hi[RW][4];
                            float o[RW][NT][4];
#pragma unroll
                            for (int r = 0; r < RW; ++r) {
                                weights(r, lo[r], hi[r]);
#pragma unroll
                                for (int n = 0; n < NT; ++n) o[r][n][0] = o[r][n][1] = o[r][n][2] = o[r][n][3] = 0.f;
                            }
#pragma unroll
                            for (int s = TERMS - 1; s >= 0; --s)
#pragma unroll
                                for (int p = 0; p < 4; p += 2)
#pragma unroll
                                    for (int r = 0; r < RW; ++r) {
                                        const uint32_t f[4] = {lo[r][p], hi[r][p], lo[r][p + 1], hi[r][p + 1]};
#pragma unroll
                                        for (int n = 0; n < NT; ++n) w4_mma(o[r][n], f, x[n][s][p], x[n][s][p + 1], Mma());
                                    }
#pragma unroll
                            for (int r = 0; r < RW; ++r)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) part[r][n][i] += o[r][n][i];
                        }
                        if (j % GS == GS - 1) {   // a group ends
                            const int gi = j / GS, from_lane = (lane & 28) | (gi & 3);
#pragma unroll
                            for (int r = 0; r < RW; ++r) {
                                const float s0 = __shfl_sync(0xffffffffu, NmType<T>::to_f(sc[r][0][gi >> 2]), from_lane);
                                const float s1 = __shfl_sync(0xffffffffu, NmType<T>::to_f(sc[r][1][gi >> 2]), from_lane);
#pragma unroll
                                for (int n = 0; n < NT; ++n)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) sum[r][n][i] = __fmaf_rn(i < 2 ? s0 : s1, part[r][n][i], sum[r][n][i]);
                            }
                        }
                    }
                }
            };
            if (steps == 8) block(std::true_type());
            else block(std::false_type());
            __syncwarp();   // the stage may be filled again
            stage = stage == STAGES - 1 ? 0 : stage + 1;
        }
        if constexpr (STAGED) {
            half ^= 1;
            if (slice + (int)ctas < slices) lay_out(half);
            __syncthreads();
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();

    // each warp's sums to its own ring, [token][row]
    float* own = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) own[(n * 8 + 2 * t + (i & 1)) * PITCH + r * 16 + g + (i >> 1) * 8] = sum[r][n][i];
    __syncthreads();
    // The block's warps are added up first, each sum where the first of them has it, then the cluster's blocks.  A thread has one row and
    // every so manieth token.
    const int rows = 16 * RW * a.row_warps, row = threadIdx.x & (rows - 1), apart = W4_THREADS / rows;
    const int tokens = d.M - m0 < NT * 8 ? (int)(d.M - m0) : NT * 8;
    const int64_t n = block_row + row;
    float* at = reinterpret_cast<float*>(w4_smem + (row / (16 * RW)) * RING) + row % (16 * RW);
    const int next_warp = a.row_warps * (RING / 4);
    const bool live = n < d.N;
    const float bias = live && d.bias ? d.bias[n] : 0.f;
    auto store = [&](int m, float y, float residual) {
        if (d.bias) y += bias;
        if (a.tab) {
            const float2 kb = a.tab->kb[nm_pwl_index(y, a.tab->inv_h, a.tab->off, (float)(a.tab->n - 1))];
            y = __fmaf_rn(kb.x, y, kb.y);
        }
        if (d.residual) y += residual;
        ((T*)d.out)[(m0 + m) * d.ldo + n] = NmType<T>::from_f(y);
    };
    auto residual_of = [&](int m) { return live && d.residual && m < tokens ? NmType<T>::to_f(((const T*)d.residual)[(m0 + m) * d.ldr + n]) : 0.f; };
#pragma unroll 4
    for (int m = threadIdx.x / rows; m < tokens; m += apart) {
        const float r = ctas == 1 ? residual_of(m) : 0.f;
        float y = at[m * PITCH];
        for (int k = 1; k < k_warps; ++k) y += at[m * PITCH + k * next_warp];
        if (ctas > 1) at[m * PITCH] = y;
        else if (live) store(m, y, r);
    }
    if (ctas == 1) return;
    nm_cluster_sync();
    if (live) {
        const uint32_t here = nm_smem_u32(at);
        for (int m = (int)rank * apart + threadIdx.x / rows; m < tokens; m += (int)ctas * apart) {
            const float r = residual_of(m);
            float v[8], y = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < (int)ctas) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c]) : "r"(nm_mapa(here + m * (PITCH * 4), c)) : "memory");
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < (int)ctas) y += v[c];
            store(m, y, r);
        }
    }
    nm_cluster_sync();   // no CTA leaves while another reads its shared memory
}

template <typename T, int NT, int RW, int GS>
nm_status launch(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    constexpr bool STAGED = NT > 1;
    constexpr int STAGES = RW == 2 ? 3 : STAGED ? 3 : 4;
    W4Args a;
    a.d = *d;
    a.tab = d->slot == NM_SLOT_NONE ? nullptr : ctx->d_tables + d->slot;
    a.k_groups = (int)(d->K / d->group);
    a.k_blocks = (int)((d->K + W4_BLOCK_K - 1) / W4_BLOCK_K);
    const int64_t token_blocks = (d->M + NT * 8 - 1) / (NT * 8), row_tiles = (d->N + 16 * RW - 1) / (16 * RW);
    const int64_t slots = (int64_t)ctx->sm_count * 2;
    // As many warps along the rows as there are; fewer (and more that split k) as long as the blocks do not fill two to an SM and every
    // warp has a block of k, and the activations' bytes that a block reads stay below the weights' (4 M / rows; STAGED: and fit).
    int rw = 8;
    while (rw > (STAGED ? 2 * NT : 1) && 16 * RW * (rw / 2) >= 4 * d->M && W4_WARPS / rw < a.k_blocks && (row_tiles + rw - 1) / rw * token_blocks < slots) rw /= 2;
    const int smem = W4_WARPS * STAGES * RW * W4_TILE + (STAGED ? 2 * (W4_WARPS / rw) * 8 * NT * W4Type<T>::TERMS * 512 : 0);
    a.row_warps = rw;
    a.row_blocks = (int)((row_tiles + rw - 1) / rw);
    const int64_t units = a.row_blocks * token_blocks;
    int ctas = 1;   // of a cluster: they split k further while there is room
    while (ctas < 8 && units * ctas * 2 <= slots && a.k_blocks >= 2 * ctas * (W4_WARPS / rw)) ctas *= 2;
    if (units * ctas > INT32_MAX) return NM_ERR_SHAPE;
    auto kernel = linear_w4_kernel<T, NT, RW, STAGES, GS>;
    static std::atomic<uint64_t> allowed{0};
    if (!nm_allow_smem(ctx, (const void*)kernel, W4_MAX_SMEM, allowed)) return NM_ERR_CUDA;
    NmLaunchScope scope(ctx, NM_KERNEL_LINEAR_W4, 0.5 * d->N * d->K, st);
    NmLaunchConfig lc(ctx, dim3((unsigned)(units * ctas)), W4_THREADS, smem, st, ctas);
    return cudaLaunchKernelEx(&lc.cfg, kernel, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

template <typename T, int GS>
nm_status by_tokens(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    // Two tiles of 16 weight rows per warp, so that each activation serves two products, where that leaves every SM two blocks' warps
    // (8 x 16384 x 8192 bf16: 35 us with one, 32 with two) and for fp32, whose terms cost most.  For more than 8 tokens one: the sums of
    // two tiles do not fit the registers.
    if (d->M <= 8) return sizeof(T) == 4 || d->N >= 32 * 2 * ctx->sm_count ? launch<T, 1, 2, GS>(ctx, d, st) : launch<T, 1, 1, GS>(ctx, d, st);
    if (d->M <= 16) return launch<T, 2, 1, GS>(ctx, d, st);
    return launch<T, 4, 1, GS>(ctx, d, st);
}
template <typename T>
nm_status dispatch(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    return d->group == 32 ? by_tokens<T, 1>(ctx, d, st) : d->group == 64 ? by_tokens<T, 2>(ctx, d, st) : by_tokens<T, 4>(ctx, d, st);
}

}  // namespace

nm_status nm_launch_linear_w4(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    switch (d->dtype) {
    case NM_F32: return dispatch<float>(ctx, d, st);
    case NM_BF16: return dispatch<__nv_bfloat16>(ctx, d, st);
    case NM_F16: return dispatch<__half>(ctx, d, st);
    default: return NM_ERR_UNSUPPORTED;
    }
}
