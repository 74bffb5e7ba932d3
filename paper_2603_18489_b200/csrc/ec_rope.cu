// ec_qk_norm_rope, ec_qk_norm_rope_paged: root-mean-square norm of every query and key head and the position rotation, one
// read and one write of each value.
//
// Bound by memory: 2 x (H_q + H_kv) x head_dim values a row (+ V, copied, in the paged form).  A head is held by
// head_dim / 16 lanes, 16 values each: the two 8-value pieces whose columns are rotated into one another (half-split
// pairs: pieces i and i + rot_dim/16; interleaved pairs stay inside a piece), so that only the sum of squares crosses lanes.
// The angles of a row are the same for all its heads: a CTA forms the rot_dim/2 sines and cosines of its rows once.
// Angle: positions[r] * inv_freq[i] in turns, in 64 bits, reduced to [-1/2, 1/2] turns there (a position of 10^5 at
// frequency 1 has 24 bits left of 41 for the fraction; fp32 would keep 7).  What fp32 cannot hold of the reduced
// angle (2^-25 of half a turn) is put back to first order: 5e-8 of an fp32 result.
// 4 x 2048 to 4096 rows of 32 + 32 heads of 128: 117 us, 5.4 TB/s; 8 x 766 to 1531 rows of 28 + 4: 38 us, 4.4 TB/s, where the
// angles and look-ups at the start of a CTA of eight rows weigh more (65 % of the issue slots).
#include "ec_common.cuh"
#include "ec_tc_ptx.cuh"

namespace ec {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 8;   // rows a CTA, at most

// 8 values as they are loaded
template <typename T>
struct Raw {
    uint4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = *(reinterpret_cast<const uint4*>(p) + i);
    }
    __device__ __forceinline__ void values(float* x) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                x[4 * i] = __uint_as_float(v[i].x), x[4 * i + 1] = __uint_as_float(v[i].y), x[4 * i + 2] = __uint_as_float(v[i].z),
                      x[4 * i + 3] = __uint_as_float(v[i].w);
        } else {
            const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
};
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
    Raw<T> r;
    r.load(p);
    r.values(x);
}
__device__ __forceinline__ void store8(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* v) {
    *reinterpret_cast<uint4*>(p) = make_uint4(tc::pack_bf16x2(v[0], v[1]), tc::pack_bf16x2(v[2], v[3]),
                                              tc::pack_bf16x2(v[4], v[5]), tc::pack_bf16x2(v[6], v[7]));
}

struct Row {       // what a CTA knows of one of its rows
    int out;       // 1: q_out (and dense k_out) are written
    long long kv;  // paged: element offset of the row's place in head 0 of its page, < 0: not written
};

template <typename T, int HD, bool kPaged>
__global__ void __launch_bounds__(kThreads, 4) rope_kernel(const RopeArgs a, int tokens) {
    constexpr int LH = HD / 16, HPB = kThreads / LH;   // lanes of a head, heads at a time
    __shared__ float2 turn[kMaxTokens][HD / 2];        // cosine, sine
    __shared__ Row rows[kMaxTokens];
    const int tid = threadIdx.x;
    const int r0 = blockIdx.x * tokens, n = min(tokens, a.n_rows - r0);
    const int half = a.d.rot_dim / 2;
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    const int hq = a.d.n_q_heads, hkv = a.d.n_kv_heads;
    const int heads = hq + hkv * (kPaged ? 2 : 1);
    const int l = tid % LH;
    // this lane's two pieces of a head
    const int pairs = a.d.rot_dim / 16;   // lanes that rotate
    const bool inter = a.d.flags & EC_ROPE_INTERLEAVED, rotates = l < pairs;
    const int c0 = rotates && !inter ? l : 2 * l, c1 = rotates && !inter ? l + pairs : 2 * l + 1;
    const bool norm = a.q_weight != nullptr;
    // The next head's loads are under way while this one is worked on, the first one's already under the angles.  (Two heads at a
    // time take 80 registers instead of 56 and with them a CTA of each SM: 45 us instead of 39 for 8 x 1531 rows, 126 instead of 121.)
    Raw<T> raw[2];
    const auto ask = [&](int item) {
        if (item >= n * heads) return;
        const int t = item / heads, h = item - t * heads;
        const long long r = r0 + t;
        const T* src = h < hq ? static_cast<const T*>(a.q) + r * a.q_stride + (long long)h * HD
                     : h < hq + hkv ? static_cast<const T*>(a.k) + r * a.k_stride + (long long)(h - hq) * HD
                                    : static_cast<const T*>(a.v) + r * a.v_stride + (long long)(h - hq - hkv) * HD;
        raw[0].load(src + c0 * 8);
        raw[1].load(src + c1 * 8);
    };
    ask(tid / LH);
    for (int i = tid; i < n * half; i += kThreads) {
        const int t = i / half, f = i % half;
        const double turns = (double)a.positions[r0 + t] * (double)a.inv_freq[f] * 0.15915494309189533577;   // / (2 pi)
        const double x = 2.0 * (turns - rint(turns));   // half turns, in [-1, 1]
        const float hi = (float)x;
        const float lo = (float)(x - (double)hi) * 3.14159265f;
        float s, c;
        sincospif(hi, &s, &c);
        turn[t][f] = make_float2(fmaf(-lo, s, c), fmaf(lo, c, s));
    }
    if (tid < n) {
        const int r = r0 + tid, pos = a.positions[r];
        Row row{pos >= 0, -1};
        if constexpr (kPaged) {
            int lo = 0, hi = a.batch;   // the sequence: the last one that starts at or before r
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.row_offsets[mid] <= r) lo = mid; else hi = mid - 1;
            }
            if (lo >= a.batch || r < a.row_offsets[0]) row.out = 0;   // padding
            if (row.out) {
                const int entry = pos / a.page_size;
                int bad = 0;
                if (entry >= a.max_pages) {
                    bad = EC_ERR_SHAPE;
                } else {
                    const int page = a.page_table[(long long)lo * a.max_pages + entry];
                    if ((unsigned)page >= (unsigned)a.n_pages) bad = EC_ERR_PAGE;
                    else row.kv = ((long long)page * a.d.n_kv_heads * a.page_size + pos % a.page_size) * HD;
                }
                if (bad && a.dev_status) atomicExch(a.dev_status, bad);
            }
        }
        rows[tid] = row;
    }
    __syncthreads();

    for (int item = tid / LH; item < n * heads; item += HPB) {
        float x[2][8];
        raw[0].values(x[0]);
        raw[1].values(x[1]);
        ask(item + HPB);
        const int t = item / heads, h = item - t * heads;
        const Row row = rows[t];
        const long long r = r0 + t;
        T* dst = nullptr;
        if (h < hq) {
            if (row.out) dst = static_cast<T*>(a.q_out) + (r * hq + h) * HD;
        } else if (h < hq + hkv) {
            if constexpr (kPaged) {
                if (row.kv >= 0) dst = static_cast<T*>(a.k_out) + row.kv + (long long)(h - hq) * a.page_size * HD;
            } else if (row.out) {
                dst = static_cast<T*>(a.k_out) + (r * hkv + h - hq) * HD;
            }
        } else if (row.kv >= 0) {
            dst = static_cast<T*>(a.v_pages) + row.kv + (long long)(h - hq - hkv) * a.page_size * HD;
        }
        if (!dst) continue;   // (the lanes of a head agree, so the reduction below stays whole within them)
        if (h < hq + hkv) {
            if (norm) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(x[0][i], x[0][i], fmaf(x[1][i], x[1][i], ss));
                const uint32_t lanes = ((1u << LH) - 1u) << ((tid & 31) / LH * LH);
#pragma unroll
                for (int o = LH / 2; o; o >>= 1) ss += __shfl_xor_sync(lanes, ss, o);
                const float inv = 1.f / sqrtf(ss * (1.f / HD) + a.d.eps);
                const T* w = static_cast<const T*>(h < hq ? a.q_weight : a.k_weight);
                float wv[2][8];
                load8(w + c0 * 8, wv[0]);
                load8(w + c1 * 8, wv[1]);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[0][i] *= inv * wv[0][i], x[1][i] *= inv * wv[1][i];
            }
            if (rotates && !inter) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 cs = turn[t][l * 8 + i];
                    const float p = x[0][i], q = x[1][i];
                    x[0][i] = fmaf(p, cs.x, -q * cs.y);
                    x[1][i] = fmaf(q, cs.x, p * cs.y);
                }
            } else if (rotates) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 cs = turn[t][l * 8 + j * 4 + i];
                        const float p = x[j][2 * i], q = x[j][2 * i + 1];
                        x[j][2 * i] = fmaf(p, cs.x, -q * cs.y);
                        x[j][2 * i + 1] = fmaf(q, cs.x, p * cs.y);
                    }
            }
        }
        store8(dst + c0 * 8, x[0]);
        store8(dst + c1 * 8, x[1]);
    }
}

template <typename T, int HD, bool kPaged>
cudaError_t launch(const RopeArgs& a, cudaStream_t stream) {
    // Few rows: one a CTA.  Many: the angles' 64-bit arithmetic and the start of a CTA are shared by several.
    int tokens = 1;
    while (tokens < kMaxTokens && (long long)a.n_rows > 8ll * sm_count() * tokens) tokens *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((a.n_rows + tokens - 1) / tokens, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, rope_kernel<T, HD, kPaged>, a, tokens);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t stream) {
    const bool bf = a.d.dtype == EC_BF16, wide = a.d.head_dim == 128, paged = a.row_offsets != nullptr;
    if (bf) {
        if (wide) return paged ? launch<__nv_bfloat16, 128, true>(a, stream) : launch<__nv_bfloat16, 128, false>(a, stream);
        return paged ? launch<__nv_bfloat16, 64, true>(a, stream) : launch<__nv_bfloat16, 64, false>(a, stream);
    }
    if (wide) return paged ? launch<float, 128, true>(a, stream) : launch<float, 128, false>(a, stream);
    return paged ? launch<float, 64, true>(a, stream) : launch<float, 64, false>(a, stream);
}

}  // namespace ec
