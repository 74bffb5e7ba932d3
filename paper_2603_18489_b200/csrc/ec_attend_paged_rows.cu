// ec_attend_paged for few query rows a kv head (decoding: one row a sequence) in bf16, and for fp32: eight or sixteen packed
// query rows a tile, the keys split over warps that know nothing of one another until the end.
//
// Bound by the K/V bytes.  A CTA's warps (four; eight or sixteen where sequences are short) take the key tiles, sixteen keys
// each: a warp loads its own chunk of K and V (rows of one page; cp.async, three stages deep, zeros behind the sequence's end, so
// that what an unfinished page holds is never multiplied), forms the scores, keeps its own running maximum and sum, and multiplies
// into its own accumulators.  Nothing but the merge at the end of a unit's keys needs the CTA together.
//   bf16   mma.sync m16n8k16 (tcgen05 has no shape below 64 rows, and this is far from bound by the tensor pipe: 7.5 % busy), P
//          rounded to bf16 for the second product as the dense kernels do (outputs are off by 2.1e-3 of their size, 1.7e-3 of it
//          their own rounding); the sums of the weights are formed from the unrounded ones
//   fp32   FMA units; a lane has one key and eight rows for the scores, HD / 32 columns of all rows for the output
// The work is cut as ec_paged.cuh says; attend_paged_combine_kernel joins the units that a cut divided.
// 32 sequences of 526 to 7892 keys, 32 heads on 8: 94 us, 5.2 TB/s (the bytes alone 76); the rest is planning (3 us), the ends of
// units (a merge of the warps, 1.5 us each) and the join.  One token over 768 keys: 10.7 us.
#include "ec_paged.cuh"
#include "ec_paged_combine.cuh"
#include "ec_tc_ptx.cuh"

namespace ec {
namespace {

using namespace paged;

constexpr int CK = 16, kMaxTM = 16;

// W warps a CTA, S stages a warp
template <typename T, int HD, int W, int S>
struct Geo {
    static constexpr int CHUNK = CK * HD * (int)sizeof(T);   // bytes of a warp's K or V chunk
    static constexpr int STAGE = 2 * CHUNK;
    static constexpr int WARP = S * STAGE;
    static constexpr int Q = sizeof(T) == 4 ? kMaxTM * HD * 4 : 0;        // fp32: the tile's query rows ...
    static constexpr int P = sizeof(T) == 4 ? W * CK * kMaxTM * 4 : 0;   // ... and the probabilities
    static constexpr int BYTES = W * WARP + Q + P;
    static constexpr int CTAS = (BYTES + 10240) * 3 <= 228 * 1024 ? 3 : (BYTES + 10240) * 2 <= 228 * 1024 ? 2 : 1;   // an SM
};

constexpr int kWholeKeys = 1024;   // room of the page table, in positions, up to which no unit is cut

struct Params {
    Plan plan;
    const void *q, *k, *v;
    void* out;
    float* partial;
    Cut* cuts;
    const int32_t* page_table;
    int page_shift, n_pages, max_pages, n_q_heads;
    float scale_log2;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool valid) {
    const uint32_t bytes = valid ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transposed(uint32_t v) {   // of an 8 x 8 tile of 16-bit values
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// A warp's state over its chunks.  Row limits: a key counts for a row while it is below lim.
// Keys and columns stand on the M axis of the products, the query rows on N, eight at a time: S^T = K Q^T and O^T = V^T P^T, so
// that eight rows, one of a token's query heads each, fill an instruction (with the rows on M it was twice as many).
template <int HD, int NT>
struct WarpBf16 {
    static constexpr int TM = 8 * NT, LD = HD + 4;   // row stride of finish(): no bank conflicts
    uint32_t qb[NT][HD / 16][2];
    float o[NT][HD / 16][4], m[NT][2], l[NT][2];      // of rows (lane % 4) * 2 + {0, 1}
    int lim[NT][2];
    __device__ __forceinline__ void start(const Params& p, const Unit& u, int lane) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int pr = u.tile * TM + nt * 8 + lane / 4, tok = pr / p.plan.group;
            const bool has = tok < u.s.n;
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q) +
                ((long long)(u.s.row0 + tok) * p.n_q_heads + u.head * p.plan.group + pr % p.plan.group) * HD + (lane & 3) * 2;
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
                for (int h = 0; h < 2; ++h) qb[nt][ks][h] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + h * 8) : 0u;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = (u.tile * TM + nt * 8 + (lane & 3) * 2 + e) / p.plan.group;
                lim[nt][e] = t < u.s.n ? limit_of(p.plan, u.s, t) : 0;
                m[nt][e] = -INFINITY;
                l[nt][e] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < HD / 16; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.f;
        }
    }
    __device__ __forceinline__ void chunk(const Params& p, uint32_t stage, int key0, int lane, const unsigned char*, float*) {
        constexpr int ROW = HD * 2;
        const int mi = lane >> 3, r = lane & 7;
        float s[NT][2][4] = {};   // even and odd steps of the columns: half the chain
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
            uint32_t a[4];
            ldsm(stage + ((mi & 1) * 8 + r) * ROW + (((ks * 2 + (mi >> 1)) ^ r) << 4), a);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma(s[nt][ks & 1], a, qb[nt][ks][0], qb[nt][ks][1]);
        }
        uint32_t pb[NT][2];
        bool moved = false;
        float f[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)   // key lane / 4 + 8 (i / 2), row (lane % 4) * 2 + i % 2
                x[i] = key0 + (lane >> 2) + (i >> 1) * 8 < lim[nt][i & 1] ? (s[nt][0][i] + s[nt][1][i]) * p.scale_log2 : -INFINITY;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float mx = fmaxf(x[e], x[2 + e]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                const float mn = fmaxf(m[nt][e], mx), ref = mn == -INFINITY ? 0.f : mn;   // (a row that sees nothing yet)
                f[nt][e] = fast_exp2(m[nt][e] - ref);
                moved |= f[nt][e] != 1.f;
                m[nt][e] = mn;
                x[e] = fast_exp2(x[e] - ref);
                x[2 + e] = fast_exp2(x[2 + e] - ref);
                l[nt][e] = fmaf(l[nt][e], f[nt][e], x[e] + x[2 + e]);   // this lane's keys alone, summed over the lanes at the end
            }
            pb[nt][0] = transposed(tc::pack_bf16x2(x[0], x[1]));
            pb[nt][1] = transposed(tc::pack_bf16x2(x[2], x[3]));
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    o[nt][i][0] *= f[nt][0], o[nt][i][1] *= f[nt][1];
                    o[nt][i][2] *= f[nt][0], o[nt][i][3] *= f[nt][1];
                }
        }
        const uint32_t vbase = stage + CK * ROW;
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) {
            uint32_t a[4];
            ldsm_t(vbase + ((mi >> 1) * 8 + r) * ROW + (((i * 2 + (mi & 1)) ^ r) << 4), a);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma(o[nt][i], a, pb[nt][0], pb[nt][1]);
        }
    }
    // un-normalised rows to dst [TM][LD], maxima and sums to ml [TM]
    __device__ __forceinline__ void finish(float* dst, float2* ml, int lane) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nt][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                const int row = nt * 8 + (lane & 3) * 2 + e;
                if (lane < 4) ml[row] = make_float2(m[nt][e], sum);
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    dst[row * LD + i * 16 + (lane >> 2)] = o[nt][i][e];
                    dst[row * LD + i * 16 + 8 + (lane >> 2)] = o[nt][i][2 + e];
                }
            }
    }
};

template <int HD>
struct WarpF32 {
    static constexpr int TM = 16, LD = HD, C = HD / 32;
    float o[TM][C], m[8], l[8];
    int lim[8];
    __device__ __forceinline__ void start(const Params& p, const Unit& u, int lane) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int tok = (u.tile * TM + (lane >> 4) * 8 + i) / p.plan.group;
            lim[i] = tok < u.s.n ? limit_of(p.plan, u.s, tok) : 0;
            m[i] = -INFINITY;
            l[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c) o[i][c] = 0.f;
    }
    __device__ __forceinline__ void chunk(const Params& p, uint32_t, int key0, int lane, const unsigned char* stage, float* qp) {
        constexpr int ROW = HD * 4;
        const float* q = qp;                                            // [TM][HD]
        float* prob = qp + TM * HD + (threadIdx.x >> 5) * CK * TM;      // [CK][TM], this warp's
        const int key = lane & 15, half = lane >> 4;
        float s[8] = {};
#pragma unroll 4
        for (int c = 0; c < HD / 4; ++c) {
            const float4 kv = *reinterpret_cast<const float4*>(stage + key * ROW + ((c ^ (key & 7)) << 4));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 qv = *reinterpret_cast<const float4*>(q + (half * 8 + i) * HD + c * 4);
                s[i] = fmaf(kv.x, qv.x, fmaf(kv.y, qv.y, fmaf(kv.z, qv.z, fmaf(kv.w, qv.w, s[i]))));
            }
        }
        float f[8];
        bool moved = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = key0 + key < lim[i] ? s[i] * p.scale_log2 : -INFINITY;
            float mx = x;
#pragma unroll
            for (int d = 8; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn;
            f[i] = exp2f(m[i] - ref);
            moved |= f[i] != 1.f;
            m[i] = mn;
            s[i] = exp2f(x - ref);
            l[i] = fmaf(l[i], f[i], s[i]);   // this lane's key alone, summed over the lanes at the end
        }
        __syncwarp();
        *reinterpret_cast<float4*>(prob + key * TM + half * 8) = make_float4(s[0], s[1], s[2], s[3]);
        *reinterpret_cast<float4*>(prob + key * TM + half * 8 + 4) = make_float4(s[4], s[5], s[6], s[7]);
        __syncwarp();
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const float g = __shfl_sync(0xffffffffu, f[i & 7], (i >> 3) * 16);
#pragma unroll
                for (int c = 0; c < C; ++c) o[i][c] *= g;
            }
        }
        const unsigned char* v = stage + CK * ROW;
#pragma unroll 4
        for (int kk = 0; kk < CK; ++kk) {
            float vv[C];
            const int byte = lane * C * 4, piece = byte >> 4;
            const unsigned char* at = v + kk * ROW + ((piece ^ (kk & 7)) << 4) + (byte & 15);
            if constexpr (C == 4) {
                const float4 x = *reinterpret_cast<const float4*>(at);
                vv[0] = x.x, vv[1] = x.y, vv[2] = x.z, vv[3] = x.w;
            } else {
                const float2 x = *reinterpret_cast<const float2*>(at);
                vv[0] = x.x, vv[1] = x.y;
            }
#pragma unroll
            for (int i4 = 0; i4 < TM / 4; ++i4) {
                const float4 pr = *reinterpret_cast<const float4*>(prob + kk * TM + i4 * 4);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    o[i4 * 4][c] = fmaf(pr.x, vv[c], o[i4 * 4][c]);
                    o[i4 * 4 + 1][c] = fmaf(pr.y, vv[c], o[i4 * 4 + 1][c]);
                    o[i4 * 4 + 2][c] = fmaf(pr.z, vv[c], o[i4 * 4 + 2][c]);
                    o[i4 * 4 + 3][c] = fmaf(pr.w, vv[c], o[i4 * 4 + 3][c]);
                }
            }
        }
    }
    __device__ __forceinline__ void finish(float* dst, float2* ml, int lane) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float sum = l[i];
#pragma unroll
            for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if ((lane & 15) == 0) ml[(lane >> 4) * 8 + i] = make_float2(m[i], sum);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c) dst[i * HD + lane * C + c] = o[i][c];
    }
};
template <typename T, int HD, int NT>
struct WarpOf { using type = WarpBf16<HD, NT>; };
template <int HD, int NT>
struct WarpOf<float, HD, NT> { using type = WarpF32<HD>; };

template <typename T, int HD, int NT, int W, int S>
__global__ void __launch_bounds__(32 * W, Geo<T, HD, W, S>::CTAS) attend_paged_rows_kernel(const Params p) {
    using G = Geo<T, HD, W, S>;
    using Warp = typename WarpOf<T, HD, NT>::type;
    constexpr int kThreads = 32 * W, TK = CK * W, kStages = S, TM = Warp::TM, LD = Warp::LD;
    static_assert(TM * LD * 4 <= G::WARP, "a warp's rows stand over its stages");
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long begin[EC_PAGED_MAX_BATCH + 1];
    __shared__ float2 ml[W][TM];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned char* mine = smem + warp * G::WARP;
    const uint32_t mine_u = tc::s2u(mine);
    float* qp = reinterpret_cast<float*>(smem + W * G::WARP);
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    lay_out(p.plan, begin);
    const long long all = begin[p.plan.batch];
    const int n = workers(p.plan, all, gridDim.x), cta = blockIdx.x;
    __shared__ long long ends[2];
    __shared__ Unit unit;
    if (warp < 2) {   // the two cuts side by side
        const Cut cut = cut_of(p.plan, begin, all, n, cta + warp, warp == 0 ? &unit : nullptr);
        if (lane == 0) ends[warp] = cut.w;
        if (threadIdx.x == 0) p.cuts[cta] = cut;
    }
    __syncthreads();
    const long long first = ends[0], last = ends[1];
    if (threadIdx.x == 0 && cta == 0) p.cuts[gridDim.x] = cut_of_end(all);

    Unit u = unit;
    for (long long w = first; w < last;) {
        if (w != first) step_unit(p.plan, u);
        const int j0 = step_at(p.plan, u, w), j1 = step_at(p.plan, u, last);
        w = min(last, u.w0 + u.steps + p.plan.start);
        const long long rows_all = (long long)u.s.n * p.plan.group;
        const int32_t* table = p.page_table + (long long)u.b * p.max_pages;
        const long long page_rows = (long long)p.plan.n_kv_heads << p.page_shift;
        // a lane's part of a chunk: 16-byte piece `piece` of rows lane / LR, + RW, ...
        constexpr int PIECES = HD * (int)sizeof(T) / 16, RW = 32 / (PIECES < 32 ? PIECES : 32), LR = PIECES < 32 ? PIECES : 32;
        auto page_at = [&](int j) -> int {
            const int key0 = j * TK + warp * CK;
            return j < j1 && key0 < u.s.kv ? table[key0 >> p.page_shift] : -1;
        };
        auto issue = [&](int j, int page) {
            if (j < j1) {
                const int key0 = j * TK + warp * CK, slot = (j - j0) % kStages;
                int valid = min(u.s.kv - key0, CK);
                if (valid > 0 && (unsigned)page >= (unsigned)p.n_pages) {
                    if (lane == 0 && p.plan.dev_status) atomicExch(p.plan.dev_status, (int)EC_ERR_PAGE);
                    valid = 0;
                }
                const long long row = (valid > 0 ? page : 0) * page_rows + ((long long)u.head << p.page_shift) + (key0 & ((1 << p.page_shift) - 1));
                const uint32_t dst = mine_u + slot * G::STAGE;
                const unsigned char* ks = static_cast<const unsigned char*>(p.k) + (valid > 0 ? row : 0) * (HD * (long long)sizeof(T));
                const unsigned char* vs = static_cast<const unsigned char*>(p.v) + (valid > 0 ? row : 0) * (HD * (long long)sizeof(T));
#pragma unroll
                for (int i = 0; i < CK / RW; ++i) {
                    const int r = i * RW + lane / LR, piece = lane % LR;
                    const bool ok = r < valid;
                    const int off = ok ? r * HD * (int)sizeof(T) + piece * 16 : 0;   // (an address inside the pool in any case)
                    const uint32_t to = dst + r * HD * (int)sizeof(T) + ((piece ^ (r & 7)) << 4);
                    cp16(to, ks + off, ok);
                    cp16(to + G::CHUNK, vs + off, ok);
                }
            }
            cp_commit();
        };
        int page = page_at(j0);
        for (int i = 0; i < kStages - 1; ++i) {
            const int next = page_at(j0 + i + 1);
            issue(j0 + i, page);
            page = next;
        }
        if constexpr (sizeof(T) == 4) {
            for (int i = threadIdx.x; i < TM * HD / 4; i += kThreads) {
                const int r = i / (HD / 4), c = i % (HD / 4), pr = u.tile * TM + r, tok = pr / p.plan.group;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (tok < u.s.n)
                    x = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) +
                        ((long long)(u.s.row0 + tok) * p.n_q_heads + u.head * p.plan.group + pr % p.plan.group) * HD + c * 4);
                *reinterpret_cast<float4*>(qp + r * HD + c * 4) = x;
            }
            __syncthreads();
        }
        Warp state;
        state.start(p, u, lane);
        for (int j = j0; j < j1; ++j) {
            const int next = page_at(j + kStages);
            issue(j + kStages - 1, page);
            page = next;
            cp_wait<kStages - 1>();
            __syncwarp();
            const int slot = (j - j0) % kStages, key0 = j * TK + warp * CK;
            if (key0 < u.s.kv) state.chunk(p, mine_u + slot * G::STAGE, key0, lane, mine + slot * G::STAGE, qp);
            __syncwarp();   // the slot is free for the load after next
        }
        cp_wait<0>();
        __syncwarp();
        state.finish(reinterpret_cast<float*>(mine), ml[warp], lane);
        __syncthreads();
        const bool whole = j0 == 0 && j1 == u.steps;
        float* part = p.partial + ((long long)cta * 2 + (j0 == 0 ? 1 : 0)) * (TM * (HD + 2));
        for (int i = threadIdx.x; i < TM * HD / 4; i += kThreads) {
            const int r = i / (HD / 4), c = i % (HD / 4) * 4;
            const long long pr = (long long)u.tile * TM + r;
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) M = fmaxf(M, ml[k][r].x);
            const float ref = M == -INFINITY ? 0.f : M;
            float acc[4] = {};
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const float f = exp2f(ml[k][r].x - ref);
                L = fmaf(f, ml[k][r].y, L);
                const float4 x = *reinterpret_cast<const float4*>(smem + k * G::WARP + (r * LD + c) * 4);
                acc[0] = fmaf(f, x.x, acc[0]), acc[1] = fmaf(f, x.y, acc[1]);
                acc[2] = fmaf(f, x.z, acc[2]), acc[3] = fmaf(f, x.w, acc[3]);
            }
            if (!whole) {
                *reinterpret_cast<float4*>(part + r * HD + c) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                if (c == 0) *reinterpret_cast<float2*>(part + TM * HD + r * 2) = make_float2(M, L);
            } else if (pr < rows_all) {
                const float inv = L > 0.f ? 1.f / L : 0.f;
                T* dst = static_cast<T*>(p.out) + ((u.s.row0 + pr / p.plan.group) * p.n_q_heads + u.head * p.plan.group + pr % p.plan.group) * HD + c;
                store4(dst, acc, inv);
            }
        }
        __syncthreads();   // before the next unit's loads and rows
    }
}

template <typename T, int HD, int NT, int W, int S>
cudaError_t launch_as(const PagedArgs& a, bool whole, cudaStream_t stream) {
    using G = Geo<T, HD, W, S>;
    Params p;
    p.plan = make_plan(a, WarpOf<T, HD, NT>::type::TM, CK * W);
    p.plan.start = 2;
    p.plan.min_steps = 4;
    p.plan.whole = whole;
    p.q = a.q, p.k = a.k_pages, p.v = a.v_pages, p.out = a.out;
    p.page_table = a.page_table;
    p.page_shift = __builtin_ctz((unsigned)a.d.page_size);
    p.n_pages = a.d.n_pages, p.max_pages = a.d.max_pages, p.n_q_heads = a.d.n_q_heads;
    p.scale_log2 = a.scale * kLog2e;
    const int ctas = sm_count() * G::CTAS;
    p.cuts = static_cast<Cut*>(a.workspace);
    p.partial = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + cuts_bytes(ctas));
    static PerDeviceOnce once;
    if (const cudaError_t e = ensure_dynamic_smem(once, attend_paged_rows_kernel<T, HD, NT, W, S>, G::BYTES); e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas, 1, 1);
    cfg.blockDim = dim3(32 * W, 1, 1);
    cfg.dynamicSmemBytes = G::BYTES;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (const cudaError_t e = cudaLaunchKernelEx(&cfg, attend_paged_rows_kernel<T, HD, NT, W, S>, p); e != cudaSuccess) return e;
    return launch_combine<T, HD>(p.plan, p.cuts, p.partial, a.out, a.d.n_q_heads, ctas, stream);
}
template <typename T, int HD>
cudaError_t launch(const PagedArgs& a, cudaStream_t stream) {
    // Short sequences: a unit is left whole to a CTA of more warps, and there is nothing to join, a launch less (one row of 28
    // heads on 4 over 768 keys 17.4 -> 14.5 us).  Not in fp32, where sixteen keys take a warp 2 us and more CTAs are worth the
    // launch (2 x 34 rows of 256 keys: 12.4 us cut, 15.4 whole).
    if constexpr (sizeof(T) == 4) {
        return launch_as<T, HD, 2, 4, 3>(a, false, stream);
    } else {
        constexpr int kWide = HD == 128 ? 8 : 16;
        const bool whole = (long long)a.d.max_pages * a.d.page_size <= kWholeKeys;
        if ((long long)a.max_rows * (a.d.n_q_heads / a.d.n_kv_heads) <= 8)
            return whole ? launch_as<T, HD, 1, kWide, 3>(a, true, stream) : launch_as<T, HD, 1, 4, 3>(a, false, stream);
        return whole ? launch_as<T, HD, 2, kWide, 3>(a, true, stream) : launch_as<T, HD, 2, 4, 3>(a, false, stream);
    }
}

}  // namespace

size_t attend_paged_rows_workspace(const ec_paged_desc& d) {
    const int ctas = sm_count() * 4;   // at most
    return cuts_bytes(ctas) + (size_t)ctas * 2 * kMaxTM * (d.head_dim + 2) * 4;
}

cudaError_t launch_attend_paged_rows(const PagedArgs& a, cudaStream_t stream) {
    if (a.d.dtype == EC_BF16)
        return a.d.head_dim == 128 ? launch<__nv_bfloat16, 128>(a, stream) : launch<__nv_bfloat16, 64>(a, stream);
    return a.d.head_dim == 128 ? launch<float, 128>(a, stream) : launch<float, 64>(a, stream);
}

}  // namespace ec
