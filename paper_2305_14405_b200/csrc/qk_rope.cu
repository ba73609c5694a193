// Norm of the heads of queries and keys (PWL rsqrt), rotation by position and write to the paged cache: one pass over the
// packed projection.  Bound by its bytes (each element is read once and written once) or, for few tokens, by latency.
// A warp goes through its units (a token, a few of its heads) with the next ones' elements on their way to a ring in shared memory; a
// lane copies what it will read itself, so there is no barrier.
#include "nm_common.cuh"

namespace {

constexpr int ROPE_WARPS = 8, ROPE_RING = 8192;   // bytes of a warp's ring: three blocks of 64 KB an SM

// groups of heads in a unit: 4 KB
template <typename T> constexpr int rope_groups() { return sizeof(T) == 4 ? 4 : 8; }

struct RopeArgs {
    nm_qk_rope_desc d;
    const NmTable* tab;
    int* status;
    int groups_q, groups_k;   // groups of 32/LPH heads that the queries and the keys make
    int slices;               // units of a token
    int to_k, to_v;           // what the keys' and the values' first element lies further than their group numbers say
    int step_t, step_slice;   // from one unit of a warp to the next
    float inv_d;
    NmDivisor by_page;
};

// Pairs of fp32 numbers in one register pair: two correctly rounded operations an instruction.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t widen(uint32_t v, __nv_bfloat16) { return nm_pack2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint64_t widen(uint32_t v, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
    return nm_pack2(f.x, f.y);
}
__device__ __forceinline__ uint32_t narrow(uint64_t v, __nv_bfloat16)
{
    float a, b;
    nm_unpack2(v, a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t narrow(uint64_t v, __half)
{
    float a, b;
    nm_unpack2(v, a, b);
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Eight channels of a head: 16 bytes of a 16-bit type, 32 of fp32.
template <typename T> struct Eight {
    static constexpr int VECS = sizeof(T) / 2;
    uint32_t raw[VECS * 4];
    __device__ __forceinline__ void load(uint32_t at)   // from the ring: 512 bytes apart
    {
#pragma unroll
        for (int i = 0; i < VECS; ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(raw[4 * i]), "=r"(raw[4 * i + 1]), "=r"(raw[4 * i + 2]), "=r"(raw[4 * i + 3])
                         : "r"(at + i * 512)
                         : "memory");
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int i = 0; i < VECS; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3]);
    }
    __device__ __forceinline__ uint64_t pair(int i) const
    {
        if constexpr (VECS == 2) return (uint64_t)raw[2 * i + 1] << 32 | raw[2 * i];
        else return widen(raw[i], T());
    }
    __device__ __forceinline__ void set(int i, uint64_t v)
    {
        if constexpr (VECS == 2) raw[2 * i] = (uint32_t)v, raw[2 * i + 1] = (uint32_t)(v >> 32);
        else raw[i] = narrow(v, T());
    }
};

__device__ __forceinline__ void load8(const float* p, float* f)
{
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}

// LPH lanes hold a head, eight channels each (lanes from d/8 on hold none), so a group of 32/LPH heads of a token is worked on at a
// time; queries, keys and values make groups of their own.  A unit is up to U groups.  With the head's reciprocal norm r a channel is
//     y_i = r * (x_i * (gamma_i c_i) + x_p * (gamma_p s_i))          (p its partner, s_i negative for the first of a pair)
// where the products with gamma serve all of the token's heads.  The partner's elements are read from the ring as they came.
// (One after another in fp32 with gamma per head: 130 instructions for 16 bytes, 111 us for 16383 tokens of 48 heads of 128 in
// bf16, whatever was in flight; so half of them.)
template <typename T, int LPH, bool PAIRS>
__global__ void __launch_bounds__(ROPE_WARPS * 32, 3) qk_rope_kernel(const RopeArgs a)
{
    const nm_qk_rope_desc& d = a.d;
    const int lane = threadIdx.x & 31, part = lane & (LPH - 1), sub = lane / LPH;
    constexpr int HPW = 32 / LPH, U = rope_groups<T>(), VECS = Eight<T>::VECS;
    const int ch = part * 8;                  // first channel of this lane
    const bool has = ch < d.d, turns = ch < d.rot;
    const int half = d.rot >> 1;
    const bool upper = !PAIRS && ch >= half;  // second channel of its pairs
    // the lane with the other channels of this lane's pairs
    const int other = PAIRS || !turns ? lane : upper ? lane - half / 8 : lane + half / 8;
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const float inv_h = a.tab->inv_h, off = a.tab->off, nm1 = (float)(a.tab->n - 1);
    const int first_k = a.groups_q, first_v = a.groups_q + a.groups_k, groups = first_v + a.groups_k;
    extern __shared__ __align__(16) unsigned char rope_smem[];
    const uint32_t ring = nm_smem_u32(rope_smem) + (threadIdx.x >> 5) * ROPE_RING;
    constexpr int STAGE = U * VECS * 512, STAGES = ROPE_RING / STAGE;
    // A unit is (t, slice); a warp's units are a grid apart.
    struct Unit {
        int t, slice;
    };
    auto advance = [&](Unit& w) {
        w.t = w.t > INT32_MAX - a.step_t - 1 ? INT32_MAX : w.t + a.step_t;
        w.slice += a.step_slice;
        if (w.slice >= a.slices) {
            w.slice -= a.slices;
            ++w.t;
        }
    };
    const int w0 = blockIdx.x * ROPE_WARPS + (threadIdx.x >> 5);
    Unit now = {w0 / a.slices, w0 % a.slices}, ahead = now, seen = now;
    // this lane's head of group number x of a token, counted within the section that begins at group number `begin`
    auto head_of = [&](int x, int begin) { return (x - begin) * HPW + sub; };
    auto fetch = [&](int stage) {
        if (ahead.t < d.T) {
            const T* row = (const T*)d.qkv + (int64_t)ahead.t * d.ld_qkv + ch;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = ahead.slice + u * a.slices, begin = x < first_k ? 0 : x < first_v ? first_k : first_v;
                if (x >= groups) break;
                if (has && head_of(x, begin) < (x < first_k ? d.heads : d.kv_heads)) {
                    const T* from = row + (x * HPW + sub) * d.d + (x < first_k ? 0 : x < first_v ? a.to_k : a.to_v);
#pragma unroll
                    for (int i = 0; i < VECS; ++i)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + stage * STAGE + (u * VECS + i) * 512 + lane * 16),
                                     "l"((const uint4*)from + i)
                                     : "memory");
                }
            }
            advance(ahead);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i) fetch(i);
    int next_slot = 0, next_pos = 0, stage = 0;
    auto look = [&] {
        if (seen.t < d.T) {
            next_slot = d.slots ? d.slots[seen.t] : 0;
            next_pos = d.rot ? d.positions[seen.t] : 0;
            advance(seen);
        }
    };
    look();
    for (; now.t < d.T; advance(now)) {
        const int64_t t = now.t;
        const int slice = now.slice, slot = next_slot, pos = next_pos;
        look();
        const bool bad_pos = d.rot && (pos < 0 || pos >= d.max_position);
        const bool bad_slot = d.k_cache && slot >= d.num_pages * d.page_size;
        if (slot >= 0 && (bad_pos || bad_slot) && lane == 0) atomicExch(a.status, (int)NM_ERR_INVALID_ARG);
        const bool skip = slot < 0 || bad_pos || bad_slot;
        const int page = d.k_cache && !skip ? a.by_page(slot) : 0;
        const int64_t at = d.k_cache ? (int64_t)page * d.stride_page + (int64_t)(slot - page * d.page_size) * d.stride_token + ch : 0;
        uint64_t c[4], s[4];   // gamma_i c_i and gamma_p s_i of the section
        int factors_of = -1;
        auto factors = [&](int section) {
            float x[8], y[8], g[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 1.f, y[i] = 0.f, g[i] = 1.f;
            if (turns) {
                const float* table = d.cos_sin + (int64_t)pos * d.rot;
                if constexpr (PAIRS) {
                    const float4 u = __ldg(reinterpret_cast<const float4*>(table + ch / 2)), v = __ldg(reinterpret_cast<const float4*>(table + half + ch / 2));
                    x[0] = x[1] = u.x, x[2] = x[3] = u.y, x[4] = x[5] = u.z, x[6] = x[7] = u.w;
                    y[1] = v.x, y[3] = v.y, y[5] = v.z, y[7] = v.w;
                    y[0] = -v.x, y[2] = -v.y, y[4] = -v.z, y[6] = -v.w;
                } else {
                    const int pair = upper ? ch - half : ch;
                    load8(table + pair, x);
                    load8(table + half + pair, y);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = upper ? y[i] : -y[i];
                }
            }
            const float* gamma = section == 0 ? d.gamma_q : d.gamma_k;
            if (gamma && has) {
                load8(gamma + ch, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= g[i];
                if (turns) {
                    if (!PAIRS) load8(gamma + (upper ? ch - half : ch + half), g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] *= PAIRS ? g[i ^ 1] : g[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = nm_pack2(x[2 * i], x[2 * i + 1]), s[i] = nm_pack2(y[2 * i], y[2 * i + 1]);
            factors_of = section;
        };
        if (!skip && slice < first_v) factors(slice >= first_k);
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();   // the lanes' copies are there
        if (!skip) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = slice + u * a.slices;
                if (x >= groups) break;
                const int section = x < first_k ? 0 : x < first_v ? 1 : 2, h = head_of(x, section == 0 ? 0 : section == 1 ? first_k : first_v);
                const bool live = has && h < (section == 0 ? d.heads : d.kv_heads);
                const uint32_t from = ring + stage * STAGE + u * VECS * 512;
                Eight<T> v;
                v.load(from + lane * 16);
                if (section == 2) {   // values are copied as they are
                    if (live && d.v_cache) v.store((T*)d.v_cache + at + (int64_t)h * d.stride_head);
                    continue;
                }
                if (section != factors_of) factors(section);
                uint64_t y[4], r2 = nm_pack2(1.f, 1.f);
                const bool norm = section == 0 ? d.gamma_q != nullptr : d.gamma_k != nullptr;
                if (norm) {
                    uint64_t q = nm_pack2(0.f, 0.f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        y[i] = v.pair(i);
                        q = fma2(y[i], y[i], q);
                    }
                    float q0, q1;
                    nm_unpack2(q, q0, q1);
                    float sq = live ? q0 + q1 : 0.f;
#pragma unroll
                    for (int o = LPH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                    const float var = __fmaf_rn(sq, a.inv_d, d.eps);
                    const float2 kb = __ldg(&a.tab->kb[nm_pwl_index(var, inv_h, off, nm1)]);
                    const float r = __fmaf_rn(kb.x, var, kb.y);
                    r2 = nm_pack2(r, r);
                }
                if (norm || d.rot) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = mul2(v.pair(i), c[i]);
                    if (d.rot && turns) {
                        if constexpr (PAIRS) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float e, o;
                                nm_unpack2(v.pair(i), e, o);
                                y[i] = fma2(nm_pack2(o, e), s[i], y[i]);
                            }
                        } else {
                            Eight<T> p;
                            p.load(from + other * 16);
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[i] = fma2(p.pair(i), s[i], y[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) v.set(i, norm ? mul2(y[i], r2) : y[i]);
                }
                if (!live) continue;
                if (section == 0) {
                    v.store((T*)d.q_out + t * d.ld_q + (int64_t)h * d.d + ch);
                } else {
                    if (d.k_out) v.store((T*)d.k_out + t * d.ld_k + (int64_t)h * d.d + ch);
                    if (d.k_cache) v.store((T*)d.k_cache + at + (int64_t)h * d.stride_head);
                }
            }
        }
        __syncwarp();   // and have been read
        fetch(stage);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <typename T>
nm_status launch(nm_ctx* ctx, const nm_qk_rope_desc* d, cudaStream_t st)
{
    const int lanes = d->d / 8, lph = lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32, hpw = 32 / lph;
    RopeArgs a;
    a.groups_q = (d->heads + hpw - 1) / hpw;
    a.groups_k = (d->kv_heads + hpw - 1) / hpw;
    const int64_t groups = a.groups_q + 2 * (int64_t)a.groups_k;
    a.inv_d = (float)(1.0 / d->d);
    a.d = *d;
    a.tab = ctx->d_tables + (d->gamma_q || d->gamma_k ? d->rsqrt_slot : 0);
    a.status = ctx->d_status;
    // A unit is up to U groups of a token's heads: fewer where there are so few tokens that the SMs' warps are not all taken.
    constexpr int U = rope_groups<T>();
    const int64_t room = (int64_t)ctx->sm_count * 3 * ROPE_WARPS;
    int64_t slices = (room + d->T - 1) / d->T;
    if (slices < (groups + U - 1) / U) slices = (groups + U - 1) / U;
    a.slices = (int)(slices > groups ? groups : slices);
    const int64_t work = (int64_t)d->T * a.slices, want = (work + ROPE_WARPS - 1) / ROPE_WARPS, cap = (int64_t)ctx->sm_count * 3;
    const int blocks = (int)(want > cap ? cap : want);
    a.step_t = blocks * ROPE_WARPS / a.slices;
    a.step_slice = blocks * ROPE_WARPS % a.slices;
    a.to_k = (d->heads - a.groups_q * hpw) * d->d;
    a.to_v = a.to_k + (d->kv_heads - a.groups_k * hpw) * d->d;
    a.by_page = NmDivisor::of(d->k_cache ? d->page_size : 1);
    NmLaunchScope scope(ctx, NM_KERNEL_QK_ROPE, 2.0 * d->T * (d->heads + 2.0 * d->kv_heads) * d->d * sizeof(T), st);
    NmLaunchConfig lc(ctx, dim3((unsigned)blocks), ROPE_WARPS * 32, ROPE_WARPS * ROPE_RING, st);
    auto kernel = d->pairs ? (lph == 8 ? qk_rope_kernel<T, 8, true> : lph == 16 ? qk_rope_kernel<T, 16, true> : qk_rope_kernel<T, 32, true>)
                           : (lph == 8 ? qk_rope_kernel<T, 8, false> : lph == 16 ? qk_rope_kernel<T, 16, false> : qk_rope_kernel<T, 32, false>);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ROPE_WARPS * ROPE_RING) != cudaSuccess) return NM_ERR_CUDA;
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
