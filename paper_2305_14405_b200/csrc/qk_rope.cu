// Norm of the heads of queries and keys (PWL rsqrt), rotation by position and write to the paged cache: one pass over the
// packed projection.  Bound by its bytes (each element is read once and written once) or, for few tokens, by latency.
#include "nm_common.cuh"

namespace {

struct RopeArgs {
    nm_qk_rope_desc d;
    const NmTable* tab;
    int* status;
    int slices;      // warps that share a token's heads
};

// Eight channels of a head: 16 bytes of a 16-bit type, 32 of fp32.
template <typename T> struct Eight {
    uint4 raw[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = raw[i];
    }
    __device__ __forceinline__ void get(float* f) const
    {
        const T* e = reinterpret_cast<const T*>(raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = NmType<T>::to_f(e[i]);
    }
    __device__ __forceinline__ void set(const float* f)
    {
        T* e = reinterpret_cast<T*>(raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = NmType<T>::from_f(f[i]);
    }
};

// LPH lanes hold a head, eight channels each (lanes from d/8 on hold none), so a warp works on 32/LPH heads of a token at a
// time.  The lane's cosines and sines serve all heads of the token.
template <typename T, int LPH>
__global__ void __launch_bounds__(256) qk_rope_kernel(const RopeArgs a)
{
    const nm_qk_rope_desc& d = a.d;
    const int lane = threadIdx.x & 31, part = lane & (LPH - 1), sub = lane / LPH;
    constexpr int HPW = 32 / LPH;
    const int ch = part * 8;                  // first channel of this lane
    const bool has = ch < d.d, turns = ch < d.rot;
    const int half = d.rot >> 1;
    const bool upper = !d.pairs && ch >= half;   // second channel of its pairs
    // the lane with the other channels of this lane's pairs
    const int other = d.pairs || !turns ? lane : upper ? lane - half / 8 : lane + half / 8;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const float inv_h = a.tab->inv_h, off = a.tab->off, nm1 = (float)(a.tab->n - 1);
    float gq[8], gk[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        gq[i] = has && d.gamma_q ? d.gamma_q[ch + i] : 0.f;
        gk[i] = has && d.gamma_k ? d.gamma_k[ch + i] : 0.f;
    }
    const int heads = d.heads + 2 * d.kv_heads;
    const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5), work = (int64_t)d.T * a.slices;
    for (int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); w < work; w += warps) {
        const int64_t t = w / a.slices;
        const int slice = (int)(w - t * a.slices);
        const int slot = d.slots ? d.slots[t] : 0;
        if (slot < 0) continue;
        const int pos = d.rot ? d.positions[t] : 0;
        const bool bad_pos = d.rot && (pos < 0 || pos >= d.max_position);
        const bool bad_slot = d.k_cache && slot >= d.num_pages * d.page_size;
        if (bad_pos || bad_slot) {
            if (lane == 0) atomicExch(a.status, (int)NM_ERR_INVALID_ARG);
            continue;
        }
        const int64_t at = d.k_cache ? (int64_t)(slot / d.page_size) * d.stride_page + (int64_t)(slot % d.page_size) * d.stride_token : 0;
        float c[8], s[8];   // of this lane's channels; the second channel of a pair takes +s, the first -s
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = d.pairs ? (ch + i) >> 1 : upper ? ch + i - half : ch + i;
            const bool second = d.pairs ? (i & 1) : upper;
            c[i] = turns ? d.cos_sin[(int64_t)pos * d.rot + pair] : 1.f;
            s[i] = turns ? d.cos_sin[(int64_t)pos * d.rot + half + pair] : 0.f;
            if (!second) s[i] = -s[i];
        }
        const T* row = (const T*)d.qkv + t * d.ld_qkv;
        for (int h0 = slice * HPW; h0 < heads; h0 += a.slices * HPW) {   // the same number of turns for all lanes
            const int h = h0 + sub;
            const bool live = h < heads && has;
            Eight<T> v;
            float f[8];
            if (live) v.load(row + (int64_t)h * d.d + ch);
            const bool is_q = h < d.heads, is_v = h >= d.heads + d.kv_heads;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 0.f;
            if (live) v.get(f);
            if (d.gamma_q || d.gamma_k) {
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sq = __fmaf_rn(f[i], f[i], sq);
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                if (is_q ? d.gamma_q != nullptr : d.gamma_k != nullptr) {
                    const float var = sq / (float)d.d + d.eps;
                    const float2 kb = a.tab->kb[nm_pwl_index(var, inv_h, off, nm1)];
                    const float r = __fmaf_rn(kb.x, var, kb.y);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = f[i] * r * (is_q ? gq[i] : gk[i]);
                }
            }
            if (d.rot) {
                float g[8];
                if (d.pairs) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = f[i ^ 1];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = __shfl_sync(0xffffffffu, f[i], other);
                }
                if (turns) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = __fmaf_rn(f[i], c[i], g[i] * s[i]);
                }
            }
            if (!live) continue;
            if (is_v) {   // values are copied as they are
                if (d.v_cache) v.store((T*)d.v_cache + at + (int64_t)(h - d.heads - d.kv_heads) * d.stride_head + ch);
                continue;
            }
            v.set(f);
            if (is_q) {
                v.store((T*)d.q_out + t * d.ld_q + (int64_t)h * d.d + ch);
            } else {
                const int hk = h - d.heads;
                if (d.k_out) v.store((T*)d.k_out + t * d.ld_k + (int64_t)hk * d.d + ch);
                if (d.k_cache) v.store((T*)d.k_cache + at + (int64_t)hk * d.stride_head + ch);
            }
        }
    }
}

template <typename T>
nm_status launch(nm_ctx* ctx, const nm_qk_rope_desc* d, cudaStream_t st)
{
    const int lanes = d->d / 8, lph = lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32, hpw = 32 / lph;
    const int heads = d->heads + 2 * d->kv_heads, groups = (heads + hpw - 1) / hpw;
    RopeArgs a;
    a.d = *d;
    a.tab = ctx->d_tables + (d->gamma_q || d->gamma_k ? d->rsqrt_slot : 0);
    a.status = ctx->d_status;
    // few tokens: a warp for every group of heads, so that the launch has one turn; many: a token per warp
    const int64_t room = (int64_t)ctx->sm_count * 32;
    int64_t slices = (room + d->T - 1) / d->T;
    a.slices = (int)(slices > groups ? groups : slices);
    const int64_t work = (int64_t)d->T * a.slices, blocks = (work + 7) / 8, cap = (int64_t)ctx->sm_count * 8;
    NmLaunchScope scope(ctx, NM_KERNEL_QK_ROPE, 2.0 * d->T * heads * d->d * sizeof(T), st);
    NmLaunchConfig lc(ctx, dim3((unsigned)(blocks > cap ? cap : blocks)), 256, 0, st);
    auto kernel = lph == 8 ? qk_rope_kernel<T, 8> : lph == 16 ? qk_rope_kernel<T, 16> : qk_rope_kernel<T, 32>;
    return cudaLaunchKernelEx(&lc.cfg, kernel, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

}  // namespace

nm_status nm_launch_qk_rope(nm_ctx* ctx, const nm_qk_rope_desc* d, cudaStream_t st)
{
    switch (d->dtype) {
    case NM_F32: return launch<float>(ctx, d, st);
    case NM_BF16: return launch<__nv_bfloat16>(ctx, d, st);
    case NM_F16: return launch<__half>(ctx, d, st);
    default: return NM_ERR_UNSUPPORTED;
    }
}
