// Joins the partial rows of the units that a cut divided (see ec_paged.cuh): the second launch of ec_attend_paged.
// CTA c looks after the cut at the start of worker c.  Where it divides a unit into P parts, the P - 1 CTAs of its cuts
// share the unit's rows; a warp takes a row: weights 2^(m_i - M) / sum, then the rows, four columns a lane.
#pragma once

#include "ec_paged.cuh"
#include "ec_tc_ptx.cuh"

namespace ec {
namespace paged {

__device__ __forceinline__ void store4(float* dst, const float* v, float f) {
    *reinterpret_cast<float4*>(dst) = make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
}
__device__ __forceinline__ void store4(__nv_bfloat16* dst, const float* v, float f) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(tc::pack_bf16x2(v[0] * f, v[1] * f), tc::pack_bf16x2(v[2] * f, v[3] * f));
}

constexpr int kCombineThreads = 256;

// partial: [worker][2 slots] of { rows [tm][HD], then (maximum, sum) [tm] }; kSwizzled: 16-byte piece c of row r at c ^ r
template <typename T, int HD, bool kSwizzled>
__global__ void __launch_bounds__(kCombineThreads) attend_paged_combine_kernel(const Plan p, const long long* cuts,
                                                                               const float* partial, T* out, int n_q_heads,
                                                                               int ctas) {
    __shared__ long long begin[EC_PAGED_MAX_BATCH + 1];
    const int c = blockIdx.x + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // (the lengths are the caller's, complete before the first launch: laid out while that one still runs)
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    const long long w = cuts[c], all = cuts[ctas];
    if (w >= all || w == cuts[c - 1]) return;   // no work behind the cut, or the same cut as the one before
    Plan quiet = p;
    quiet.dev_status = nullptr;
    lay_out(quiet, begin);
    const Unit u = unit_at(quiet, begin, w);
    if (w == u.w0) return;   // between two units
    const long long end = u.w0 + u.steps;
    int lo = c, hi = c;      // cuts inside the unit; part i runs from cut i to cut i + 1
    while (cuts[lo - 1] > u.w0) --lo;
    while (hi + 1 <= ctas && cuts[hi + 1] < end) ++hi;
    const int sharers = hi - lo + 1, parts = sharers + 1;
    const long long rows = min((long long)p.tm, (long long)u.s.n * p.group - (long long)u.tile * p.tm);
    const long long stride = (long long)p.tm * (HD + 2);
    // part 0 is the worker of the cut before `lo`, its second slot
    auto part_at = [&](int i) { return partial + ((long long)(lo - 1 + i) * 2 + (i == 0 ? 1 : 0)) * stride; };
    for (long long r = (c - lo) + (long long)warp * sharers; r < rows; r += (long long)sharers * (kCombineThreads / 32)) {
        float M = -INFINITY;
        for (int i = lane; i < parts; i += 32) M = fmaxf(M, part_at(i)[p.tm * HD + r * 2]);
        M = tc::redux_max(M);
        const float ref = M == -INFINITY ? 0.f : M;
        float L = 0.f, acc[HD / 32] = {};
        for (int i0 = 0; i0 < parts; i0 += 32) {
            float f = 0.f;
            if (i0 + lane < parts) {
                const float2 ml = *reinterpret_cast<const float2*>(part_at(i0 + lane) + p.tm * HD + r * 2);
                f = exp2f(ml.x - ref);
                L = fmaf(f, ml.y, L);
            }
            const int here = min(32, parts - i0);
#pragma unroll 4
            for (int i = 0; i < here; ++i) {
                const float g = __shfl_sync(0xffffffffu, f, i);
                constexpr int PIECES = HD / 4;
                int at = lane * (HD / 32);
                if constexpr (kSwizzled) at = (((at >> 2) ^ ((int)r & (PIECES - 1))) << 2) | (at & 3);
                const float* src = part_at(i0 + i) + r * HD + at;
                if constexpr (HD == 128) {
                    const float4 x = *reinterpret_cast<const float4*>(src);
                    acc[0] = fmaf(g, x.x, acc[0]), acc[1] = fmaf(g, x.y, acc[1]);
                    acc[2] = fmaf(g, x.z, acc[2]), acc[3] = fmaf(g, x.w, acc[3]);
                } else {
                    const float2 x = *reinterpret_cast<const float2*>(src);
                    acc[0] = fmaf(g, x.x, acc[0]), acc[1] = fmaf(g, x.y, acc[1]);
                }
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
        const float inv = L > 0.f ? 1.f / L : 0.f;
        const long long pr = (long long)u.tile * p.tm + r;
        T* dst = out + ((u.s.row0 + pr / p.group) * n_q_heads + u.head * p.group + pr % p.group) * HD + lane * (HD / 32);
        if constexpr (HD == 128) {
            store4(dst, acc, inv);
        } else if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float2*>(dst) = make_float2(acc[0] * inv, acc[1] * inv);
        } else {
            *reinterpret_cast<uint32_t*>(dst) = tc::pack_bf16x2(acc[0] * inv, acc[1] * inv);
        }
    }
}

inline size_t cuts_bytes(int ctas) { return ((size_t)(ctas + 1) * 8 + 127) & ~(size_t)127; }

inline Plan make_plan(const PagedArgs& a, int tm, int tk) {
    Plan p;
    p.row_offsets = a.row_offsets;
    p.kv_lens = a.kv_lens;
    p.batch = a.d.batch;
    p.n_rows = a.n_rows;
    p.max_rows = a.max_rows;
    const long long most = (long long)a.d.max_pages * a.d.page_size;
    p.max_kv = (int)(most < 0x7fffff00ll ? most : 0x7fffff00ll);
    p.group = a.d.n_q_heads / a.d.n_kv_heads;
    p.n_kv_heads = a.d.n_kv_heads;
    p.mask_block = a.d.mask_block;
    p.tm = tm;
    p.tk = tk;
    p.min_steps = 1;
    p.dev_status = a.dev_status;
    return p;
}

template <typename T, int HD, bool kSwizzled = false>
cudaError_t launch_combine(const Plan& p, const long long* cuts, const float* partial, void* out, int n_q_heads, int ctas,
                           cudaStream_t stream) {
    if (ctas < 2) return cudaSuccess;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas - 1, 1, 1);
    cfg.blockDim = dim3(kCombineThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_paged_combine_kernel<T, HD, kSwizzled>, p, cuts, partial, static_cast<T*>(out), n_q_heads, ctas);
}

}  // namespace paged
}  // namespace ec
