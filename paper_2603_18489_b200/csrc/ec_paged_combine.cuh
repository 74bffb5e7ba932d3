// Joins the partial rows of the units that a cut divided (see ec_paged.cuh): the second launch of ec_attend_paged.
// CTA c looks after the cut at the start of worker c.  Where it divides a unit into P parts, the P - 1 CTAs of its cuts
// share the unit's rows: weights 2^(m_i - M) / sum first, then the rows.
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

constexpr int kCombineThreads = 512;
constexpr int kMaxWeights = 2048;   // 2 x 256, and 256 + 2 x the parts (at most one a CTA)

// partial: [worker][2 slots] of { rows [tm][HD], then (maximum, sum) [tm] }; kColumns: the rows of every 128 as [HD / 4][128][4]
template <typename T, int HD, bool kColumns>
__global__ void __launch_bounds__(kCombineThreads) attend_paged_combine_kernel(const Plan p, const Cut* cuts,
                                                                               const float* partial, T* out, int n_q_heads,
                                                                               int ctas) {
    // rows / (parts - 1), rounded up, times parts: most for two parts of 256 rows, or one row of as many parts as there are CTAs
    __shared__ float weight[kMaxWeights];
    __shared__ int run[2];
    const int c = blockIdx.x + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    const Cut u = cuts[c];
    if (u.w0 < 0 || u.w == u.w0) return;   // nothing behind the cut, or it stands between two units
    // the cuts that divide the same unit are the CTAs' around this one: warp 0 looks down, warp 1 up
    if (warp < 2) {
        const int step = warp == 0 ? -1 : 1;
        int at = c;
        for (;;) {
            const int i = at + step * (lane + 1);
            const bool same = i >= 1 && i <= ctas && cuts[i].w0 == u.w0 && cuts[i].w > u.w0;
            const uint32_t m = __ballot_sync(0xffffffffu, same);
            at += step * (m == 0xffffffffu ? 32 : __ffs(~m) - 1);
            if (m != 0xffffffffu) break;
        }
        if (lane == 0) run[warp] = at;
    }
    __syncthreads();
    const int lo = run[0], hi = run[1];   // part i runs from cut lo - 1 + i to the next
    const int sharers = hi - lo + 1, parts = sharers + 1;
    const int rows = (int)min((long long)p.tm, (long long)u.n * p.group - (long long)u.tile * p.tm);
    const long long stride = (long long)p.tm * (HD + 2);
    // part 0 is the worker of the cut before `lo`, its second slot
    auto part_at = [&](int i) { return partial + ((long long)(lo - 1 + i) * 2 + (i == 0 ? 1 : 0)) * stride; };
    const int per = (rows + sharers - 1) / sharers, row0 = (c - lo) * per, mine = min(per, rows - row0);
    // the weights of this CTA's rows, one row a thread
    for (int i = threadIdx.x; i < mine; i += kCombineThreads) {
        const long long at = (long long)p.tm * HD + (row0 + i) * 2;
        float M = -INFINITY, L = 0.f;
#pragma unroll 4
        for (int k = 0; k < parts; ++k) M = fmaxf(M, part_at(k)[at]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll 4
        for (int k = 0; k < parts; ++k) {
            const float2 ml = *reinterpret_cast<const float2*>(part_at(k) + at);
            const float f = exp2f(ml.x - ref);
            L = fmaf(f, ml.y, L);
            weight[i * parts + k] = f;
        }
        const float inv = L > 0.f ? 1.f / L : 0.f;
        for (int k = 0; k < parts; ++k) weight[i * parts + k] *= inv;
    }
    __syncthreads();
    if constexpr (kColumns) {
        // Eight rows and 64 columns a warp, a lane sixteen columns of a row: its four loads of a part are 128 contiguous bytes of
        // eight lanes, its two stores a sector.  (A row a warp, as below: 32 lines a load, 256 rows over 4096 keys 59 us a
        // call, 47 like this.)
        for (int item = warp; item < (mine + 7) / 8 * (HD / 64); item += kCombineThreads / 32) {
            const int i = item / (HD / 64) * 8 + (lane & 7), r = row0 + min(i, mine - 1), piece = item % (HD / 64) * 16 + (lane >> 3) * 4;
            const long long off = (((r >> 7) * (HD / 4) + piece) * 128 + (r & 127)) * 4;
            float acc[16] = {};
#pragma unroll 2
            for (int k = 0; k < parts; ++k) {
                const float* src = part_at(k) + off;
                float4 x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const float4*>(src + e * 512);
                const float f = weight[min(i, mine - 1) * parts + k];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[4 * e] = fmaf(f, x[e].x, acc[4 * e]), acc[4 * e + 1] = fmaf(f, x[e].y, acc[4 * e + 1]);
                    acc[4 * e + 2] = fmaf(f, x[e].z, acc[4 * e + 2]), acc[4 * e + 3] = fmaf(f, x[e].w, acc[4 * e + 3]);
                }
            }
            if (i >= mine) continue;
            const long long pr = (long long)u.tile * p.tm + r;
            T* dst = out + ((u.row0 + pr / p.group) * n_q_heads + u.head * p.group + pr % p.group) * HD + piece * 4;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float* v = acc + 8 * e;
                *reinterpret_cast<uint4*>(dst + 8 * e) = make_uint4(tc::pack_bf16x2(v[0], v[1]), tc::pack_bf16x2(v[2], v[3]),
                                                                    tc::pack_bf16x2(v[4], v[5]), tc::pack_bf16x2(v[6], v[7]));
            }
        }
        return;
    }
    // the rows, four at a time a warp: their loads are under way together
    constexpr int C = HD / 32, RG = 4;
    for (int i0 = warp * RG; i0 < mine; i0 += kCombineThreads / 32 * RG) {
        float acc[RG][C] = {};
#pragma unroll 2
        for (int k = 0; k < parts; ++k) {
            const float* src = part_at(k) + (long long)row0 * HD + lane * C;
            float x[RG][C];
#pragma unroll
            for (int j = 0; j < RG; ++j) {
                const float* at = src + min(i0 + j, mine - 1) * HD;
                if constexpr (HD == 128) {
                    const float4 v = *reinterpret_cast<const float4*>(at);
                    x[j][0] = v.x, x[j][1] = v.y, x[j][2] = v.z, x[j][3] = v.w;
                } else {
                    const float2 v = *reinterpret_cast<const float2*>(at);
                    x[j][0] = v.x, x[j][1] = v.y;
                }
            }
#pragma unroll
            for (int j = 0; j < RG; ++j) {
                const float f = weight[min(i0 + j, mine - 1) * parts + k];
#pragma unroll
                for (int e = 0; e < C; ++e) acc[j][e] = fmaf(f, x[j][e], acc[j][e]);
            }
        }
#pragma unroll
        for (int j = 0; j < RG; ++j) {
            if (i0 + j >= mine) break;
            const long long pr = (long long)u.tile * p.tm + row0 + i0 + j;
            T* dst = out + ((u.row0 + pr / p.group) * n_q_heads + u.head * p.group + pr % p.group) * HD + lane * C;
            if constexpr (HD == 128) {
                store4(dst, acc[j], 1.f);
            } else if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<float2*>(dst) = make_float2(acc[j][0], acc[j][1]);
            } else {
                *reinterpret_cast<uint32_t*>(dst) = tc::pack_bf16x2(acc[j][0], acc[j][1]);
            }
        }
    }
}

inline size_t cuts_bytes(int ctas) { return ((size_t)(ctas + 1) * sizeof(Cut) + 127) & ~(size_t)127; }

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
    p.start = 0;
    p.whole = 0;
    p.min_steps = 1;
    p.dev_status = a.dev_status;
    return p;
}

template <typename T, int HD, bool kColumns = false>
cudaError_t launch_combine(const Plan& p, const Cut* cuts, const float* partial, void* out, int n_q_heads, int ctas,
                           cudaStream_t stream) {
    if (ctas < 2 || p.whole) return cudaSuccess;
    if (2 * 256 + 2 * ctas > kMaxWeights) return cudaErrorInvalidValue;   // (a GPU of more than 256 SMs)
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas - 1, 1, 1);
    cfg.blockDim = dim3(kCombineThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_paged_combine_kernel<T, HD, kColumns>, p, cuts, partial, static_cast<T*>(out), n_q_heads, ctas);
}

}  // namespace paged
}  // namespace ec
