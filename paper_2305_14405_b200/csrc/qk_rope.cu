// Norm of the heads of queries and keys (PWL rsqrt), rotation by position and write to the paged cache: one pass over the
// packed projection.  Each element is read once and written once, rounded once at the end; sums and rotation are fp32.
// Measured: 16383 tokens of 48 heads of 128 in bf16 (407 MB), half of the channels turned in neighbouring pairs 87 us, 4.7 TB/s, all of them
// turned in halves 101 us; 192 tokens 4.4 us; one token 3.0 us, all of it latency.
// Large cases issue about 0.57 instructions per cycle and scheduler with half of the DRAM rate taken: the partner's piece is read and widened a second
// time when halves turn, values pass through registers, and where a group holds more heads than there are key heads its lanes idle (9899
// tokens of 8 + 2 heads of 128: 32 us for 10 of bytes).  Without norm and rotation the same moves take 70 to 75 us.
// A warp goes through its units (a token, a few of its heads) with the next ones' elements on their way to a ring in shared memory; a
// lane copies what it will read itself, so there is no barrier.
#include <type_traits>

#include "nm_common.cuh"

namespace {

constexpr int ROPE_WARPS = 8, ROPE_RING = 12288;   // bytes of a warp's ring: two blocks of 96 KB an SM

// groups of heads in a unit: 4 KB
template <typename T> constexpr int rope_groups() { return sizeof(T) == 4 ? 2 : 4; }

struct RopeArgs {
    nm_qk_rope_desc d;
    const NmTable* tab;
    int* status;
    int groups_q, groups_k;   // groups of 32/LPH heads that the queries and the keys make
    int lanes;                // lanes of a head, two pieces each
    int slices, per;          // units of a token, groups of a unit
    int to_k, to_v;           // what the keys' and the values' first element lies further than their group numbers say
    int step_t, step_slice;   // from one unit of a warp to the next
    float inv_d;
    NmDivisor by_page;
};

__device__ __forceinline__ float2 widen(uint32_t v, __nv_bfloat16) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ float2 widen(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ uint32_t narrow(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t narrow(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Eight channels of a head: 16 bytes of a 16-bit type, 32 of fp32.
template <typename T> struct Piece {
    static constexpr int VECS = sizeof(T) / 2, BYTES = VECS * 16;
    uint32_t raw[VECS * 4];
    __device__ __forceinline__ void load(uint32_t at)
    {
#pragma unroll
        for (int i = 0; i < VECS; ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(raw[4 * i]), "=r"(raw[4 * i + 1]), "=r"(raw[4 * i + 2]), "=r"(raw[4 * i + 3])
                         : "r"(at + i * 16)
                         : "memory");
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int i = 0; i < VECS; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3]);
    }
    __device__ __forceinline__ void get(float* f) const
    {
        if constexpr (VECS == 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(raw[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 x = widen(raw[i], T());
                f[2 * i] = x.x, f[2 * i + 1] = x.y;
            }
        }
    }
    __device__ __forceinline__ void set(const float* f)
    {
        if constexpr (VECS == 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[i] = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = narrow(f[2 * i], f[2 * i + 1], T());
        }
    }
};
template <typename T> __device__ __forceinline__ void rope_copy(uint32_t dst, const T* src)
{
#pragma unroll
    for (int i = 0; i < Piece<T>::VECS; ++i)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i * 16), "l"((const uint4*)src + i) : "memory");
}

__device__ __forceinline__ void load8(const float* p, float* f)
{
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}

// LPH lanes hold a head, two pieces of eight channels each (pieces part and part + lanes; some have one or none), so a group of 32/LPH
// heads of a token is worked on at a time; queries, keys and values make groups of their own.  A unit is up to U neighbouring groups.
// With the head's reciprocal norm r a channel is
//     y_i = r * (x_i * (gamma_i c_i) + x_p * (gamma_p s_i))          (p its partner, s_i negative for the first of a pair)
// where the products with gamma serve all of the token's heads.  The partner's elements are read from the ring as they came.
template <typename T, int LPH, bool PAIRS>
__global__ void __launch_bounds__(ROPE_WARPS * 32, 2) qk_rope_kernel(const RopeArgs a)
{
    const nm_qk_rope_desc& d = a.d;
    using P = Piece<T>;
    const int lane = threadIdx.x & 31, part = lane & (LPH - 1), sub = lane / LPH;
    constexpr int HPW = 32 / LPH, U = rope_groups<T>(), GROUP = 64 * P::BYTES, STAGE = U * GROUP, STAGES = ROPE_RING / STAGE;
    const int half = d.rot >> 1;
    extern __shared__ __align__(16) unsigned char rope_smem[];
    const uint32_t ring = nm_smem_u32(rope_smem) + (threadIdx.x >> 5) * ROPE_RING;
    // The lane's pieces: first channel, whether there is one, whether it turns and is the second of its pairs, place in a group and
    // that of its partner's piece.
    int ch[2];
    bool has[2], turns[2], upper[2];
    uint32_t place[2], partner[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int piece = part + k * a.lanes;
        ch[k] = piece * 8;
        has[k] = part < a.lanes && ch[k] < d.d;
        turns[k] = has[k] && ch[k] < d.rot;
        upper[k] = !PAIRS && ch[k] >= half;
        const int other = PAIRS || !turns[k] ? piece : upper[k] ? piece - half / 8 : piece + half / 8;
        place[k] = (sub * 2 * LPH + piece) * P::BYTES;
        partner[k] = (sub * 2 * LPH + other) * P::BYTES;
    }
    nm_grid_launch_dependents();
    nm_grid_dependency_wait();
    const float inv_h = a.tab->inv_h, off = a.tab->off, nm1 = (float)(a.tab->n - 1);
    const int first_k = a.groups_q, first_v = a.groups_q + a.groups_k, groups = first_v + a.groups_k;
    const bool even = a.to_k == 0 && a.to_v == 0;   // every group is full
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
            const int x0 = ahead.slice * a.per, n = min(a.per, groups - x0);
            const T* row = (const T*)d.qkv + (int64_t)ahead.t * d.ld_qkv + (x0 * HPW + sub) * d.d;
            const uint32_t to = ring + stage * STAGE;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= n) break;
                bool live = true;
                const T* from = row;
                if (!even) {
                    const int x = x0 + u, begin = x < first_k ? 0 : x < first_v ? first_k : first_v;
                    live = head_of(x, begin) < (x < first_k ? d.heads : d.kv_heads);
                    from += x < first_k ? 0 : x < first_v ? a.to_k : a.to_v;
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (live && has[k]) rope_copy<T>(to + u * GROUP + place[k], from + ch[k]);
                row += HPW * d.d;
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
        const int x0 = now.slice * a.per, n = min(a.per, groups - x0), slot = next_slot, pos = next_pos;
        look();
        const bool bad_pos = d.rot && (pos < 0 || pos >= d.max_position);
        const bool bad_slot = d.k_cache && slot >= d.num_pages * d.page_size;
        if (slot >= 0 && (bad_pos || bad_slot) && lane == 0) atomicExch(a.status, (int)NM_ERR_INVALID_ARG);
        const bool skip = slot < 0 || bad_pos || bad_slot;
        float c[2][8], s[2][8];   // gamma_i c_i and gamma_p s_i of the section
        int factors_of = -1;
        auto factors = [&](int section) {
            const float* gamma = section == 0 ? d.gamma_q : d.gamma_k;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float *x = c[k], *y = s[k], g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 1.f, y[i] = 0.f, g[i] = 1.f;
                if (turns[k]) {
                    const float* table = d.cos_sin + (int64_t)pos * d.rot;
                    if constexpr (PAIRS) {
                        const float4 u = __ldg(reinterpret_cast<const float4*>(table + ch[k] / 2)), v = __ldg(reinterpret_cast<const float4*>(table + half + ch[k] / 2));
                        x[0] = x[1] = u.x, x[2] = x[3] = u.y, x[4] = x[5] = u.z, x[6] = x[7] = u.w;
                        y[1] = v.x, y[3] = v.y, y[5] = v.z, y[7] = v.w;
                        y[0] = -v.x, y[2] = -v.y, y[4] = -v.z, y[6] = -v.w;
                    } else {
                        const int pair = upper[k] ? ch[k] - half : ch[k];
                        load8(table + pair, x);
                        load8(table + half + pair, y);
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = upper[k] ? y[i] : -y[i];
                    }
                }
                if (gamma && has[k]) {
                    load8(gamma + ch[k], g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= g[i];
                    if (turns[k]) {
                        if (!PAIRS) load8(gamma + (upper[k] ? ch[k] - half : ch[k] + half), g);
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] *= PAIRS ? g[i ^ 1] : g[i];
                    }
                }
            }
            factors_of = section;
        };
        T *q_row = nullptr, *k_row = nullptr, *k_at = nullptr, *v_at = nullptr;
        if (!skip) {
            if (x0 < first_v) factors(x0 >= first_k);
            q_row = (T*)d.q_out + t * d.ld_q;
            k_row = d.k_out ? (T*)d.k_out + t * d.ld_k : nullptr;
            if (d.k_cache) {
                const int page = a.by_page(slot);
                const int64_t at = (int64_t)page * d.stride_page + (int64_t)(slot - page * d.page_size) * d.stride_token;
                k_at = (T*)d.k_cache + at;
                v_at = (T*)d.v_cache + at;
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();   // the lanes' copies are there
        if (!skip) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= n) break;
                const int x = x0 + u;
                const int section = x < first_k ? 0 : x < first_v ? 1 : 2, h = head_of(x, section == 0 ? 0 : section == 1 ? first_k : first_v);
                const bool live = even || h < (section == 0 ? d.heads : d.kv_heads);
                const uint32_t from = ring + stage * STAGE + u * GROUP;
                P v[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) v[k].load(from + place[k]);
                if (section == 2) {   // values are copied as they are
                    if (live && v_at) {
                        T* to = v_at + (int64_t)h * d.stride_head;
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            if (has[k]) v[k].store(to + ch[k]);
                    }
                    continue;
                }
                if (section != factors_of) factors(section);
                const bool norm = section == 0 ? d.gamma_q != nullptr : d.gamma_k != nullptr;
                if (norm || d.rot) {
                    float y[2][8], z[2][8], r = 1.f;
#pragma unroll
                    for (int k = 0; k < 2; ++k) v[k].get(y[k]);
                    if (norm) {
                        float sq[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            sq[i & 1] = __fmaf_rn(y[0][i], y[0][i], sq[i & 1]);
                            sq[2 + (i & 1)] = __fmaf_rn(y[1][i], y[1][i], sq[2 + (i & 1)]);
                        }
                        r = (live && has[0] ? sq[0] + sq[1] : 0.f) + (live && has[1] ? sq[2] + sq[3] : 0.f);
#pragma unroll
                        for (int o = LPH / 2; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) z[k][i] = y[k][i] * c[k][i];
                        if (turns[k]) {
                            float p[8];
                            if constexpr (PAIRS) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) p[i] = y[k][i ^ 1];
                            } else {
                                P w;
                                w.load(from + partner[k]);
                                w.get(p);
                            }
#pragma unroll
                            for (int i = 0; i < 8; ++i) z[k][i] = __fmaf_rn(p[i], s[k][i], z[k][i]);
                        }
                    }
                    if (norm) {
                        const float var = __fmaf_rn(r, a.inv_d, d.eps);
                        const float2 kb = __ldg(&a.tab->kb[nm_pwl_index(var, inv_h, off, nm1)]);
                        r = __fmaf_rn(kb.x, var, kb.y);
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int i = 0; i < 8; ++i) z[k][i] *= r;
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) v[k].set(z[k]);
                }
                if (!live) continue;
                T* to = section == 0 ? q_row + h * d.d : k_row ? k_row + h * d.d : k_at + (int64_t)h * d.stride_head;
                if (section == 1 && !k_row && !k_at) continue;
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (has[k]) v[k].store(to + ch[k]);
                if (section == 1 && k_row && k_at) {
                    to = k_at + (int64_t)h * d.stride_head;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (has[k]) v[k].store(to + ch[k]);
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
    const int lanes = (d->d / 8 + 1) / 2, lph = lanes <= 4 ? 4 : lanes <= 8 ? 8 : 16, hpw = 32 / lph;
    RopeArgs a;
    a.groups_q = (d->heads + hpw - 1) / hpw;
    a.groups_k = (d->kv_heads + hpw - 1) / hpw;
    const int64_t groups = a.groups_q + 2 * (int64_t)a.groups_k;
    a.lanes = lanes;
    a.inv_d = (float)(1.0 / d->d);
    a.d = *d;
    a.tab = ctx->d_tables + (nm_qk_rope_norms(d) ? d->rsqrt_slot : 0);
    a.status = ctx->d_status;
    // A unit is up to U groups of a token's heads: fewer where there are so few tokens that the SMs' warps are not all taken, but not so few
    // that some warps get a second unit (700 tokens, 32 + 8 heads of 128, bf16: 10.5 us with 2800 units for 2368 warps, 6.9 with 2100).
    constexpr int U = rope_groups<T>();
    const int64_t room = (int64_t)ctx->sm_count * 2 * ROPE_WARPS;
    int64_t slices = room / d->T;
    if (slices < (groups + U - 1) / U) slices = (groups + U - 1) / U;
    a.per = (int)((groups + slices - 1) / slices);
    a.slices = (int)((groups + a.per - 1) / a.per);
    const int64_t work = (int64_t)d->T * a.slices, want = (work + ROPE_WARPS - 1) / ROPE_WARPS, cap = (int64_t)ctx->sm_count * 2;
    const int blocks = (int)(want > cap ? cap : want);
    a.step_t = blocks * ROPE_WARPS / a.slices;
    a.step_slice = blocks * ROPE_WARPS % a.slices;
    a.to_k = (d->heads - a.groups_q * hpw) * d->d;
    a.to_v = a.to_k + (d->kv_heads - a.groups_k * hpw) * d->d;
    a.by_page = NmDivisor::of(d->k_cache ? d->page_size : 1);
    NmLaunchScope scope(ctx, NM_KERNEL_QK_ROPE, 2.0 * d->T * (d->heads + 2.0 * d->kv_heads) * d->d * sizeof(T), st);
    NmLaunchConfig lc(ctx, dim3((unsigned)blocks), ROPE_WARPS * 32, ROPE_WARPS * ROPE_RING, st);
    auto kernels = [&](auto turn) {   // by the lanes of a head
        constexpr bool PAIRS = decltype(turn)::value;
        return lph == 4 ? qk_rope_kernel<T, 4, PAIRS> : lph == 8 ? qk_rope_kernel<T, 8, PAIRS> : qk_rope_kernel<T, 16, PAIRS>;
    };
    auto kernel = d->pairs ? kernels(std::true_type()) : kernels(std::false_type());
    static std::atomic<uint64_t> allowed[6];
    if (!nm_allow_smem(ctx, (const void*)kernel, ROPE_WARPS * ROPE_RING, allowed[(lph == 4 ? 0 : lph == 8 ? 1 : 2) + (d->pairs ? 3 : 0)])) return NM_ERR_CUDA;
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
