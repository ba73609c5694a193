// Few tokens times 4-bit weights with group scales, PWL epilogue.
//
// Bound by the weights' bytes as long as the tokens are few.  The weights are the row operand of m16n8k16 products (16 weight rows, 8
// tokens, nothing padded but the last tokens), their codes made 16-bit numbers in registers: a word of eight codes gives pairs
// (k, k + 4) by one mask each, 128 + c (bf16) or 1024 + c (fp16) by the bits, c - 8 by one exact subtraction, so products and their
// sums within a group are those of whole numbers and activations; the group's sum takes its scale in fp32.  tcgen05 would want the
// 16-bit weights written to tensor or shared memory first, four times the bytes that arrive, and a drain per group.
// fp32 activations are three bf16 terms (8 + 8 + 8 bits: exact), three products each.
//
// Every warp streams its own weights through a ring of asynchronous copies (256 codes of 16 or 32 rows a stage, so 128 bytes a row):
// no barrier in the loop.  Activations come through L1, shared by the warps of a block that work on the same k.
#include "nm_common.cuh"

namespace {

constexpr int W4_WARPS = 8, W4_THREADS = W4_WARPS * 32, W4_BLOCK_K = 256, W4_TILE = 2048;   // a stage of 16 rows: 128 bytes each

struct W4Args {
    nm_linear_w4_desc d;
    const NmTable* tab;
    int row_warps, k_blocks, row_blocks;
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

// Codes i and i + 4 of a word as a pair of whole numbers -8..7.
__device__ __forceinline__ uint32_t w4_pair(uint32_t w, int i, __nv_bfloat16)
{
    const uint32_t v = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;   // 128 + c
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), __floats2bfloat162_rn(136.f, 136.f));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t w4_pair(uint32_t w, int i, __half)
{
    const uint32_t v = ((w >> (4 * i)) & 0x000f000fu) | 0x64006400u;   // 1024 + c
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&v), __floats2half2_rn(1032.f, 1032.f));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Eight activations of one token as pairs (i, i + 4), for every term.
template <typename T> struct W4Acts {
    static constexpr int TERMS = W4Type<T>::TERMS;
    uint32_t p[TERMS][4];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int s = 0; s < TERMS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) p[s][i] = 0;
    }
    __device__ __forceinline__ void load(const T* x)
    {
        if constexpr (TERMS == 1) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(x));
            p[0][0] = __byte_perm(v.x, v.z, 0x5410);
            p[0][1] = __byte_perm(v.x, v.z, 0x7632);
            p[0][2] = __byte_perm(v.y, v.w, 0x5410);
            p[0][3] = __byte_perm(v.y, v.w, 0x7632);
        } else {
            const float4 lo = __ldg(reinterpret_cast<const float4*>(x)), hi = __ldg(reinterpret_cast<const float4*>(x) + 1);
            const float a[4] = {lo.x, lo.y, lo.z, lo.w}, b[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t ta[3], tb[3];
                split(a[i], ta);
                split(b[i], tb);
#pragma unroll
                for (int s = 0; s < 3; ++s) p[s][i] = __byte_perm(ta[s], tb[s], 0x7632);
            }
        }
    }
    // x as three bf16 numbers in the upper halves: the first two cut off (so none of them overflows), the rest has 8 bits left.
    // What is not finite stays in the first term alone (an infinity's rest would be NaN).
    static __device__ __forceinline__ void split(float x, uint32_t* t)
    {
        const uint32_t bits = __float_as_uint(x);
        if ((bits & 0x7f800000u) == 0x7f800000u) {
            t[0] = (bits & 0x007fffffu) ? 0x7fc00000u : bits;
            t[1] = t[2] = 0;
            return;
        }
        t[0] = bits & 0xffff0000u;
        const float r = x - __uint_as_float(t[0]);
        t[1] = __float_as_uint(r) & 0xffff0000u;
        t[2] = __float_as_uint(r - __uint_as_float(t[1])) & 0xffff0000u;
    }
};

template <int BYTES> __device__ __forceinline__ void w4_copy(uint32_t dst, const void* src, bool valid)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(valid ? BYTES : 0) : "memory");
}

// NT tiles of 8 tokens, RW tiles of 16 weight rows per warp.  row_warps warps of a block lie along the rows, the others and the
// CTAs of a cluster split k, block by block in turn; their sums are added in that order at the end.
template <typename T, int NT, int RW, int STAGES>
__global__ void __launch_bounds__(W4_THREADS, 2) linear_w4_kernel(const W4Args a)
{
    using Mma = typename W4Type<T>::Mma;
    constexpr int TERMS = W4Type<T>::TERMS, RING = STAGES * RW * W4_TILE, PITCH = 16 * RW + 4;
    static_assert(NT * 8 * PITCH * 4 <= RING, "a warp's sums fit its ring");
    extern __shared__ __align__(128) unsigned char w4_smem[];
    const nm_linear_w4_desc& d = a.d;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int row_warp = warp % a.row_warps, k_warp = warp / a.row_warps, k_warps = W4_WARPS / a.row_warps;
    uint32_t ctas;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t rank = nm_cluster_ctarank();
    const int64_t unit = blockIdx.x / ctas;
    const int64_t m0 = unit / a.row_blocks * (NT * 8), block_row = unit % a.row_blocks * (16 * RW * a.row_warps);
    const int64_t n0 = block_row + row_warp * (16 * RW);
    const int step = k_warps * (int)ctas, first = (int)rank * k_warps + k_warp;
    unsigned char* ring = w4_smem + warp * RING;
    const uint32_t ring_at = nm_smem_u32(ring);
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();

    const int copy_row = lane >> 3, copy_chunk = lane & 7;
    auto fetch = [&](int b, int stage) {
        if (b < a.k_blocks) {
            const int64_t at = (int64_t)b * (W4_BLOCK_K / 2) + copy_chunk * 16;
            const bool in_k = at * 2 < d.K;
#pragma unroll
            for (int r = 0; r < RW * 4; ++r) {
                const int row = r * 4 + copy_row;   // 16-byte piece c of a row lies at place c ^ (row & 7): word reads hit all banks
                const bool valid = in_k && n0 + row < d.N;
                w4_copy<16>(ring_at + stage * (RW * W4_TILE) + row * 128 + ((copy_chunk ^ (row & 7)) << 4),
                            valid ? d.codes + (n0 + row) * d.ld_codes + at : d.codes, valid);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float sum[RW][NT][4], part[RW][NT][4];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[r][n][i] = part[r][n][i] = 0.f;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(first + s * step, s);

    const int groups = W4_BLOCK_K / d.group, flush = d.group / 32 - 1;   // groups of a block; a group ends where (j & flush) == flush
    const T* scales = (const T*)d.scales;
    const T* acts[NT];
    bool token[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        token[n] = m0 + n * 8 + g < d.M;
        acts[n] = (const T*)d.A + (token[n] ? (m0 + n * 8 + g) * d.lda : 0) + t * 8;
    }
    int stage = 0;
    for (int b = first; b < a.k_blocks; b += step) {
        fetch(b + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
        // scales of groups t and t + 4 of the block, of rows g and g + 8; handed round among four lanes below
        float sc[RW][2][2];
#pragma unroll
        for (int r = 0; r < RW; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int64_t row = n0 + r * 16 + h * 8 + g;
                    const int gi = t + 4 * q;
                    const int64_t at = (int64_t)b * groups + gi;
                    sc[r][h][q] = gi < groups && at * d.group < d.K && row < d.N ? NmType<T>::to_f(scales[row * d.ld_scales + at]) : 0.f;
                }
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();
        const unsigned char* tile = ring + stage * (RW * W4_TILE);
        const int64_t k0 = (int64_t)b * W4_BLOCK_K;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (k0 + j * 32 < d.K) {   // the same for the whole warp: K is a multiple of 32
                W4Acts<T> x[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    x[n].zero();
                    if (token[n]) x[n].load(acts[n] + k0 + j * 32);
                }
#pragma unroll
                for (int r = 0; r < RW; ++r) {
                    const uint32_t w0 = *reinterpret_cast<const uint32_t*>(tile + (r * 16 + g) * 128 + ((j ^ g) << 4) + t * 4);
                    const uint32_t w1 = *reinterpret_cast<const uint32_t*>(tile + (r * 16 + g + 8) * 128 + ((j ^ g) << 4) + t * 4);
#pragma unroll
                    for (int p = 0; p < 4; p += 2) {
                        const uint32_t f[4] = {w4_pair(w0, p, Mma()), w4_pair(w1, p, Mma()), w4_pair(w0, p + 1, Mma()), w4_pair(w1, p + 1, Mma())};
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int s = 0; s < TERMS; ++s) w4_mma(part[r][n], f, x[n].p[s][p], x[n].p[s][p + 1], Mma());
                    }
                }
                if ((j & flush) == flush) {
                    const int gi = j / (flush + 1), from = (lane & 28) | (gi & 3);
#pragma unroll
                    for (int r = 0; r < RW; ++r) {
                        const float s0 = __shfl_sync(0xffffffffu, gi < 4 ? sc[r][0][0] : sc[r][0][1], from);
                        const float s1 = __shfl_sync(0xffffffffu, gi < 4 ? sc[r][1][0] : sc[r][1][1], from);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                sum[r][n][i] = __fmaf_rn(i < 2 ? s0 : s1, part[r][n][i], sum[r][n][i]);
                                part[r][n][i] = 0.f;
                            }
                    }
                }
            }
        }
        __syncwarp();   // the stage may be filled again
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();

    // each warp's sums to its own ring, [token][row]
    float* mine = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(n * 8 + 2 * t + (i & 1)) * PITCH + r * 16 + g + (i >> 1) * 8] = sum[r][n][i];
    if (ctas > 1) nm_cluster_sync();
    else __syncthreads();
    const int rows = 16 * RW * a.row_warps;
    for (int x = (int)rank * W4_THREADS + threadIdx.x; x < rows * NT * 8; x += (int)ctas * W4_THREADS) {
        const int row = x % rows, m = x / rows;
        const int64_t n = block_row + row, tok = m0 + m;
        if (n >= d.N || tok >= d.M) continue;
        const int at = (row / (16 * RW)) * RING + (m * PITCH + row % (16 * RW)) * 4;
        float y = 0.f;
        for (uint32_t c = 0; c < ctas; ++c) {
            const uint32_t base = nm_mapa(nm_smem_u32(w4_smem + at), c);
            for (int k = 0; k < k_warps; ++k) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(base + k * a.row_warps * RING) : "memory");
                y += v;
            }
        }
        if (d.bias) y += d.bias[n];
        if (a.tab) {
            const float2 kb = a.tab->kb[nm_pwl_index(y, a.tab->inv_h, a.tab->off, (float)(a.tab->n - 1))];
            y = __fmaf_rn(kb.x, y, kb.y);
        }
        if (d.residual) y += NmType<T>::to_f(((const T*)d.residual)[tok * d.ldr + n]);
        ((T*)d.out)[tok * d.ldo + n] = NmType<T>::from_f(y);
    }
    if (ctas > 1) nm_cluster_sync();   // no CTA leaves while another reads its shared memory
}

template <typename T, int NT, int RW>
nm_status launch(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    constexpr int STAGES = RW == 1 ? 4 : 3, SMEM = W4_WARPS * STAGES * RW * W4_TILE;
    W4Args a;
    a.d = *d;
    a.tab = d->slot == NM_SLOT_NONE ? nullptr : ctx->d_tables + d->slot;
    a.k_blocks = (int)((d->K + W4_BLOCK_K - 1) / W4_BLOCK_K);
    const int64_t token_blocks = (d->M + NT * 8 - 1) / (NT * 8), row_tiles = (d->N + 16 * RW - 1) / (16 * RW);
    // A block reads its tokens' activations once for all its rows: as many rows as keep those bytes below the weights' (4 M / rows).
    // Below that, fewer row warps (and more that split k) as long as the blocks do not fill two to an SM and every warp has a block of k.
    const int64_t tokens = d->M < NT * 8 ? d->M : NT * 8, slots = (int64_t)ctx->sm_count * 2;
    int rw = 8;
    while (rw > 1 && 16 * RW * (rw / 2) >= 4 * tokens && W4_WARPS / rw < a.k_blocks && (row_tiles + rw - 1) / rw * token_blocks < slots) rw /= 2;
    a.row_warps = rw;
    a.row_blocks = (int)((row_tiles + rw - 1) / rw);
    const int64_t units = a.row_blocks * token_blocks;
    int ctas = 1;   // of a cluster: they split k further while there is room
    while (ctas < 8 && units * ctas * 2 <= slots && a.k_blocks >= 2 * ctas * (W4_WARPS / rw)) ctas *= 2;
    if (units * ctas > INT32_MAX) return NM_ERR_SHAPE;
    auto kernel = linear_w4_kernel<T, NT, RW, STAGES>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess) return NM_ERR_CUDA;
    NmLaunchScope scope(ctx, NM_KERNEL_LINEAR_W4, 0.5 * d->N * d->K, st);
    NmLaunchConfig lc(ctx, dim3((unsigned)(units * ctas)), W4_THREADS, SMEM, st, ctas);
    return cudaLaunchKernelEx(&lc.cfg, kernel, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

template <typename T>
nm_status dispatch(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    // one tile of weight rows per warp where the activations are few beside them, two otherwise (each then serves two products)
    if (d->M <= 8) return launch<T, 1, sizeof(T) == 4 ? 2 : 1>(ctx, d, st);
    if (d->M <= 16) return launch<T, 2, 2>(ctx, d, st);
    return launch<T, 4, 2>(ctx, d, st);
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
