// Few tokens times 4-bit weights with group scales, PWL epilogue.
#include "nm_common.cuh"

namespace {

struct W4Args {
    nm_linear_w4_desc d;
    const NmTable* tab;
};

// A warp per output column and four tokens, the lanes along K.
template <typename T>
__global__ void __launch_bounds__(128) linear_w4_kernel(const W4Args a)
{
    const nm_linear_w4_desc& d = a.d;
    const int lane = threadIdx.x & 31;
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), m0 = (int64_t)blockIdx.y * 4;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    if (n >= d.N) return;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t k = lane * 8; k < d.K; k += 256) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(d.codes + n * d.ld_codes + k / 2);
        const float s = NmType<T>::to_f(((const T*)d.scales)[n * d.ld_scales + k / d.group]);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m0 + m >= d.M) continue;
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x = __fmaf_rn((float)((int)(w >> (4 * i) & 15) - 8), NmType<T>::to_f(((const T*)d.A)[(m0 + m) * d.lda + k + i]), x);
            acc[m] = __fmaf_rn(s, x, acc[m]);
        }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[m] += __shfl_xor_sync(0xffffffffu, acc[m], o);
        if (lane == 0 && m0 + m < d.M) {
            float y = acc[m] + (d.bias ? d.bias[n] : 0.f);
            if (a.tab) {
                const float2 kb = a.tab->kb[nm_pwl_index(y, a.tab->inv_h, a.tab->off, (float)(a.tab->n - 1))];
                y = __fmaf_rn(kb.x, y, kb.y);
            }
            if (d.residual) y += NmType<T>::to_f(((const T*)d.residual)[(m0 + m) * d.ldr + n]);
            ((T*)d.out)[(m0 + m) * d.ldo + n] = NmType<T>::from_f(y);
        }
    }
}

template <typename T>
nm_status launch(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    const int64_t bx = (d->N + 3) / 4, by = (d->M + 3) / 4;
    if (by > 65535) return NM_ERR_SHAPE;
    W4Args a;
    a.d = *d;
    a.tab = d->slot == NM_SLOT_NONE ? nullptr : ctx->d_tables + d->slot;
    NmLaunchScope scope(ctx, NM_KERNEL_LINEAR_W4, 0.5 * d->N * d->K, st);
    NmLaunchConfig lc(ctx, dim3((unsigned)bx, (unsigned)by), 128, 0, st);
    return cudaLaunchKernelEx(&lc.cfg, linear_w4_kernel<T>, a) == cudaSuccess ? NM_OK : NM_ERR_CUDA;
}

}  // namespace

nm_status nm_launch_linear_w4(nm_ctx* ctx, const nm_linear_w4_desc* d, cudaStream_t st)
{
    switch (d->dtype) {
    case NM_F32: return launch<float>(ctx, d, st);
    case NM_BF16: return launch<__nv_bfloat16>(ctx, d, st);
    case NM_F16: return launch<__half>(ctx, d, st);
    default: return NM_ERR_UNSUPPORTED;
    }
}
