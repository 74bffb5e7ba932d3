// ec_attend_paged for more than sixteen packed query rows a kv head (chunked prefill, blocks of mask tokens), bf16: the
// Blackwell tensor cores, keys and values by TMA page by page.
//
// Bound by the tensor pipe and the exponentials where rows are many, by the K/V bytes where they are few.  One persistent
// CTA an SM takes its stretch of the line of units (ec_paged.cuh): a unit is two tiles of 128 packed query rows of one kv head
// over key tiles of 128.  The body is that of the dense kernel (ec_attend_dense_tc.cu, where its choices are measured):
//   warp 0      TMA producer: a key tile is 128 / page_size pages, each one box a 64-column half (one box for both where a
//               page is a whole tile); pages wholly behind the sequence's end are not asked for
//   warp 1      tcgen05.mma issuer: S_t = Q_t K^T, O_t += P_t V with P in tensor memory
//   warps 2-17  softmax, four warpgroups: (row tile) x (64-column half); no running maximum in the first pass, a row's
//               reference is its largest score among the first eight keys of the part that it sees.  They also bring Q into
//               shared memory (packed rows are rows of several heads and tokens: plain loads, the swizzle by hand)
// P is rounded to bf16: tcgen05 takes both operands in one type, and a second product for what is left would be half as much work
// again; sums of the weights are formed from the unrounded ones.  Outputs are off by 2.3e-3 of their size, 1.7e-3 of it their own rounding.
// The issuer zeroes the rows of the last V tile that stand behind the sequence's end (an unfinished page may hold anything, and
// 0 x NaN is NaN).  A row sees keys below its limit; a tile whose keys are below the lowest limit of a warp's rows needs no mask.
// The roles go from unit to unit by themselves: the producer, which is ahead of the others, writes down what the next unit is
// (four places, B_SEGFULL and B_SEGFREE), barriers and ring go on, and so the next unit's keys are on their way while this one's
// rows are still written (us, barriers set up anew for each unit / like this: 4096 causal rows with 32 heads on 8 227 / 164;
// chunks of 1100 to 1330 rows 215 / 206).  A unit that a cut divides leaves its un-normalised rows in the workspace, columns by
// fours with the row fastest, as the threads hold them, for the second launch to join.
// 4 x 2048 rows over 8192 keys each, 32 heads on 8: 855 us, 1.13 PFLOP/s (power-capped); 4096 rows over as many keys, 32 heads: 263 us
// (the dense kernel, whose caches are one piece and whose last wave is cut by the host: 198); chunks of 1100 to 1330 rows over
// 1105 to 3746 keys: 220 us, 815 TFLOP/s of the pairs that are seen.
#include "ec_paged.cuh"
#include "ec_paged_combine.cuh"
#include "ec_tc_ptx.cuh"

namespace ec {
namespace {

using namespace tc;
using namespace paged;

constexpr int BM = 128, BN = 128;
constexpr int kSoftThreads = 512, kThreads = 64 + kSoftThreads;
constexpr uint32_t SUB = 128 * 128;   // [128 rows x 64 bf16], 128-byte swizzle: 16 KB
constexpr int kSlots = 5;
constexpr int kSegments = 4;
struct Segment {   // what the roles know of the unit at hand
    Unit u;
    int j0, j1;    // key tiles of this CTA
    int more;      // 0: nothing left
};
template <int HD>
struct Geo {
    static constexpr uint32_t TILE = HD / 64 * SUB;
    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_RING = 2 * TILE;
    static constexpr uint32_t OFF_BAR = OFF_RING + kSlots * TILE;
    static constexpr uint32_t OFF_SEG = OFF_BAR + 256;
    static constexpr uint32_t OFF_XCH = OFF_SEG + 256;
    static constexpr uint32_t NEEDED = OFF_XCH + 2 * 2 * BM * 4;
    static constexpr uint32_t BYTES = HD == 128 ? 232448 : NEEDED + 1024;
    static_assert(kSegments * sizeof(Segment) <= 256 && NEEDED + 256 <= BYTES, "shared memory");
    static_assert((EC_PAGED_MAX_BATCH + 1) * 8 <= kSlots * TILE, "what stands over the ring at the start");
};
constexpr uint32_t TM_COLS = 512;
constexpr uint32_t TM_S = 0, TM_O = 256;

enum { B_FULL = 0, B_FREE = kSlots, B_SFULL = B_FREE + 3, B_PFULL = B_SFULL + 2, B_PVDONE = B_PFULL + 4,
       B_QFULL = B_PVDONE + 2, B_VERDICT = B_QFULL + 2, B_SEGFULL = B_VERDICT + 1, B_SEGFREE = B_SEGFULL + kSegments,
       B_COUNT = B_SEGFREE + kSegments };
static_assert(B_COUNT * 8 + 24 <= 256, "barriers and flags");

constexpr float kMaxSum = 1.152921504606846976e18f;   // 2^60

struct Params {
    Plan plan;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* partial;
    Cut* cuts;
    const int32_t* page_table;
    int page_shift, n_pages, max_pages, n_q_heads;
    float scale_log2;
};

__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
// packed rows of a unit
__device__ __forceinline__ int rows_of(const Plan& p, const Unit& u) {
    return (int)min((long long)u.s.n * p.group - (long long)u.tile * (2 * BM), (long long)(2 * BM));
}
// Where packed row r of a unit stands: token of the sequence, query head.  Made anew where it is needed: kept, it would cost
// the softmax registers.
struct Places {
    int group, tok0, head0, row0, head;
    __device__ __forceinline__ Places(const Plan& p, const Unit& unit) {
        const volatile Unit& u = unit;
        group = p.group;
        const long long first = (long long)u.tile * (2 * BM);
        tok0 = (int)(first / group);
        head0 = (int)(first - (long long)tok0 * group);
        row0 = u.s.row0;
        head = u.head;
    }
    __device__ __forceinline__ int token(int r) const { return tok0 + (head0 + r) / group; }
    __device__ __forceinline__ long long element(int r, int n_q_heads, int hd) const {   // of q and out
        const unsigned pr = head0 + r, tok = pr / (unsigned)group, hh = pr - tok * group;
        return ((long long)(row0 + tok0 + (int)tok) * n_q_heads + head * group + (int)hh) * hd;
    }
};

// what the roles need of a unit
struct Job {
    int j0, T, kv, rows, n_tiles_q;   // first key tile, key tiles, keys of the sequence, packed rows, row tiles
    // One row tile: the two halves of the CTA take its even and its odd key tiles, each with a reference and an accumulator of
    // its own, so that the softmax of one tile runs under the products of the other; the rows are joined at the end.
    bool split;
    __device__ __forceinline__ Job(const Plan& p, const Segment& seg)
        : j0(uniform(seg.j0)), T(uniform(seg.j1) - j0), kv(uniform(seg.u.s.kv)), rows(uniform(rows_of(p, seg.u))),
          n_tiles_q(rows > BM ? 2 : 1), split(n_tiles_q == 1 && T > 1) {}
};

template <int HD>
__global__ void __launch_bounds__(kThreads, 1)
attend_paged_tiles_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Params p) {
    constexpr uint32_t TILE = Geo<HD>::TILE, OFF_Q = Geo<HD>::OFF_Q, OFF_RING = Geo<HD>::OFF_RING, OFF_BAR = Geo<HD>::OFF_BAR,
                       OFF_XCH = Geo<HD>::OFF_XCH;
    constexpr int CW = HD / 2, CH = CW / 8, HALVES = HD / 64;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (s2u(smem_raw) + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - s2u(smem_raw));
    const uint32_t bars = base + OFF_BAR;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gbase + OFF_BAR + B_COUNT * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(gbase + OFF_BAR + B_COUNT * 8 + 4);
    volatile int* again = reinterpret_cast<volatile int*>(gbase + OFF_BAR + B_COUNT * 8 + 8);   // [2], by unit
    volatile int* go = again + 2;   // [2], by unit
    Segment* segments = reinterpret_cast<Segment*>(gbase + Geo<HD>::OFF_SEG);   // [kSegments]
    float* xch = reinterpret_cast<float*>(gbase + OFF_XCH);
    int32_t* const dev_status = p.plan.dev_status;
    auto bar = [&](int idx) { return bars + idx * 8; };
    if (base - s2u(smem_raw) + Geo<HD>::NEEDED > Geo<HD>::BYTES) {   // never with the 1024-byte alignment the runtime gives
        if (threadIdx.x == 0 && dev_status) atomicExch(dev_status, (int)EC_ERR_CUDA);
        return;
    }
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, cta = blockIdx.x;

    if (tid == 0) {
        prefetch_map(&map_k);
        prefetch_map(&map_v);
        for (int i = 0; i < B_COUNT; ++i)
            mbar_init(bar(i), (i >= B_PFULL && i < B_PFULL + 4) || (i >= B_QFULL && i < B_QFULL + 2) ? 256u : i >= B_SEGFREE ? 17u : 1u);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *abort_flag = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s2u(tmem_slot)), "r"(TM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    pdl_wait();
    pdl_launch_dependents();
    // ---- this CTA's stretch of the line (the layout stands over the ring until the first unit starts) ----
    long long last;
    {
        long long* begin = reinterpret_cast<long long*>(gbase + OFF_RING);
        lay_out(p.plan, begin);
        const long long all = begin[p.plan.batch];
        const int n = workers(p.plan, all, gridDim.x);
        long long* ends = reinterpret_cast<long long*>(xch);
        if (warp < 2) {   // the two cuts side by side
            const Cut cut = cut_of(p.plan, begin, all, n, cta + warp, warp == 0 ? &segments[0].u : nullptr);
            if (lane == 0) ends[warp] = cut.w;
            if (tid == 0) p.cuts[cta] = cut;
        }
        __syncthreads();
        const long long first = ends[0];
        last = ends[1];
        if (tid == 0) {
            Segment& s = segments[0];
            s.more = first < last;
            s.j0 = step_at(p.plan, s.u, first);
            s.j1 = step_at(p.plan, s.u, last);
            if (cta == 0) p.cuts[gridDim.x] = cut_of_end(all);
            mbar_arrive(bar(B_SEGFULL));
        }
    }
    fence_async_smem();   // the ring is the TMA's from here on
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;

    // (values out of shared memory are not warp-uniform to the compiler, and then neither is anything in a loop over them: see
    // elect_one on what that costs the issuer; for the same reason each role has its loop over the units and its state to itself)
    if (warp == 0) {
        // ================================ TMA producer ======================================
        // ring slot, the group that frees it and the phase of that barrier; ring entries so far, as far as they matter
        int slot = 0, group_free = 0, entries = 0;
        uint32_t turn = 0;
        for (int it = 0;; ++it) {
            const Segment& seg = segments[it % kSegments];
            mbar_wait_warp(bar(B_SEGFULL + it % kSegments), (it / kSegments) & 1, abort_flag, dev_status);
            if (*abort_flag || !uniform(seg.more)) break;
            const Job job(p.plan, seg);
            const int j0 = job.j0, T = job.T, kv = job.kv;
            const bool split = job.split;
            const bool elected = elect_one();
            const int32_t* table = p.page_table + (long long)seg.u.b * p.max_pages;
            const int ps = 1 << p.page_shift, boxes_page = ps == BN ? 1 : HALVES;
            const int pg = lane / boxes_page, half = lane % boxes_page;   // this lane's box of a tile
            int bad = 0;
            auto page_of = [&](int j) -> int {
                const int key = (j0 + j) * BN + pg * ps;
                if (j >= T || pg * ps >= BN || key >= kv) return -1;
                const int page = table[key >> p.page_shift];
                if ((unsigned)page < (unsigned)p.n_pages) return page;
                bad = 1;
                return 0;   // (something of the pool)
            };
            // Ring entries, from 2T on those of the second pass: K_0 V_0 K_1 V_1 ..., with split K_0 K_1 V_0 K_2 V_1 ... V_T-2 V_T-1.
            // A K tile's pages are looked up one K tile ahead; those of the V tiles to come are kept: one, with split
            // that of the tile before too.
            int ahead = page_of(0), kept = -1, kept_next = -1;
            for (int n = 0; n < 4 * T; ++n) {
                if (n == 2 * T) {
                    // the next unit, for all
                    const int nx = (it + 1) % kSegments;
                    if (it + 1 >= kSegments) mbar_wait_warp(bar(B_SEGFREE + nx), ((it + 1) / kSegments - 1) & 1, abort_flag, dev_status);
                    if (*abort_flag) break;   // (nothing is written over while somebody may read it)
                    if (lane == 0) {
                        Segment s = seg;
                        s.more = s.u.w0 + s.u.steps + p.plan.start < last;
                        if (s.more) {
                            step_unit(p.plan, s.u);
                            s.j0 = 0;
                            s.j1 = step_at(p.plan, s.u, last);
                        }
                        segments[nx] = s;
                        mbar_arrive(bar(B_SEGFULL + nx));
                    }
                    __syncwarp();
                    mbar_wait_warp(bar(B_VERDICT), it & 1, abort_flag, dev_status);
                    if (!again[it & 1]) break;
                    ahead = page_of(0);
                }
                const int m = n >= 2 * T ? n - 2 * T : n;
                bool is_v = m & 1;
                int j = m >> 1;
                if (split && m > 0) {
                    is_v = !(m & 1) || m == 2 * T - 1;
                    j = m == 2 * T - 1 ? T - 1 : is_v ? (m - 2) >> 1 : (m + 1) >> 1;
                }
                int page;
                if (is_v) {
                    page = kept;
                    kept = kept_next;
                } else {
                    page = ahead;
                    if (split && j > 0) kept_next = page;   // (V_j-1 is still to come)
                    else kept = page;
                    ahead = page_of(j + 1);
                }
                // (entries of all units count: an even number each)
                if (entries + n > kSlots && !(n & 1) && ++group_free == 3) group_free = 0, turn ^= 1;
                if (entries + n >= kSlots) mbar_wait_warp(bar(B_FREE + group_free), turn, abort_flag, dev_status);
                const int keys = min(max(kv - (j0 + j) * BN, 0), BN), pages = (keys + ps - 1) >> p.page_shift;
                if (elected) mbar_expect_tx(bar(B_FULL + slot), (uint32_t)(pages << p.page_shift) * (HD * 2));
                __syncwarp();
                if (page >= 0)
                    tma_load_4d(base + OFF_RING + slot * TILE + half * SUB + pg * ps * 128, is_v ? &map_v : &map_k, 0, 0, half,
                                page * p.plan.n_kv_heads + seg.u.head, bar(B_FULL + slot));
                __syncwarp();
                if (++slot == kSlots) slot = 0;
            }
            entries = min(entries + (uniform(again[it & 1]) ? 4 : 2) * T, 2 * kSlots);   // (even, and more than the ring holds)
            if (__any_sync(0xffffffffu, bad) && elected && dev_status) atomicExch(dev_status, (int)EC_ERR_PAGE);
            __syncwarp();
        }
    } else if (warp == 1) {
        // ================================ MMA issuer ========================================
        // ring slot and phase of the next tile, the next group to release; by row tile, the phases of P and of Q
        int slot = 0, group_free = 0;
        uint32_t phase = 0, p_phase = 0, q_phase = 0;
        for (int it = 0;; ++it) {
            const Segment& seg = segments[it % kSegments];
            mbar_wait_warp(bar(B_SEGFULL + it % kSegments), (it / kSegments) & 1, abort_flag, dev_status);
            if (*abort_flag || !uniform(seg.more)) break;
            const Job job(p.plan, seg);
            const int j0 = job.j0, T = job.T, kv = job.kv, n_tiles_q = job.n_tiles_q;
            const bool split = job.split;
            // the tile that the sequence ends inside of, counted from j0; T or more: not here
            const int j_end = (kv & (BN - 1)) || kv == 0 ? kv / BN - j0 : T;
            const bool elected = elect_one();
            constexpr uint32_t IDESC_S = instr_desc(BN, 0), IDESC_PV = instr_desc(HD, 1);
            const uint64_t desc_q = smem_desc(base + OFF_Q, 16, 1024);
            auto scores = [&](int t, uint64_t desc_rows, uint64_t desc_k, int k0, int k1) {
                if (elected) {
#pragma unroll
                    for (int k = k0; k < k1; ++k) {
                        const uint32_t koff = ((k >> 2) * SUB + (k & 3) * 32) / 16;
                        mma_ss(tmem + TM_S + t * 128, desc_rows + koff, desc_k + koff, IDESC_S, k > 0);
                    }
                }
            };
            auto products_s = [&](int t, uint64_t desc_k, int k0, int k1) { scores(t, desc_q + t * (TILE / 16), desc_k, k0, k1); };
            // P V of part h of the probabilities: the first 48 keys of each half of the tile, then the others
            auto outputs = [&](int t, uint64_t desc_v, int h, bool add) {
                if (elected) {
#pragma unroll
                    for (int i = 0; i < 6; ++i) {
                        if (h && i >= 2) break;
                        const int k = h ? i * 4 + 3 : (i / 3) * 4 + i % 3;
                        mma_ts(tmem + TM_O + t * HD, tmem + TM_S + t * 128 + (k >> 2) * 64 + (k & 3) * 8, desc_v + k * 128, IDESC_PV,
                               add || k > 0);
                    }
                }
            };
            // a V tile that the sequence ends in has landed: rows behind the end become zero
            auto zeroed = [&](int slot_v) {
                unsigned char* v = gbase + OFF_RING + slot_v * TILE;
                for (int i = (kv - (j0 + j_end) * BN) * 8 + lane; i < BN * 8; i += 32)
#pragma unroll
                    for (int hf = 0; hf < HALVES; ++hf) *reinterpret_cast<uint4*>(v + hf * SUB + i * 16) = make_uint4(0, 0, 0, 0);
                fence_async_smem();
                __syncwarp();
            };
            auto full = [&](int ahead) {
                const bool wrapped = slot + ahead >= kSlots;
                return mbar_test(bar(B_FULL + slot + ahead - (wrapped ? kSlots : 0)), phase ^ (wrapped ? 1u : 0u));
            };
            auto take = [&](bool landed) {
                if (!landed) mbar_wait_warp(bar(B_FULL + slot), phase, abort_flag, dev_status);
                const int s = slot;
                if (++slot == kSlots) slot = 0, phase ^= 1;
                return s;
            };
            auto release = [&]() {
                if (elected) commit(bar(B_FREE + group_free));
                if (++group_free == 3) group_free = 0;
            };
            constexpr int kPeek = HD / 16 - 2;
            for (int pass = 0; pass < 2; ++pass) {
                if (pass == 1) {
                    mbar_wait_warp(bar(B_VERDICT), it & 1, abort_flag, dev_status);
                    if (!again[it & 1]) break;
                }
                if (split) {
                    for (int t = 0; t < 2; ++t) {   // both chains have Q_0
                        const uint64_t desc_k = smem_desc(base + OFF_RING + take(false) * TILE, 16, 1024);
                        mbar_wait_warp(bar(B_QFULL), q_phase & 1, abort_flag, dev_status);
                        fence_after();
                        scores(t, desc_q, desc_k, 0, HD / 16);
                        if (elected) commit(bar(B_SFULL + t));
                        if (t == 0) release();
                    }
                    for (int j = 0; j < T; ++j) {
                        const int t = j & 1;
                        const int slot_v = take(false);
                        const uint64_t desc_v = smem_desc(base + OFF_RING + slot_v * TILE, SUB, 1024);
                        if (j == j_end) zeroed(slot_v);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            mbar_wait_warp(bar(B_PFULL + h * 2 + t), (p_phase >> t) & 1, abort_flag, dev_status);
                            fence_after();
                            outputs(t, desc_v, h, j > 1);
                        }
                        p_phase ^= 1u << t;
                        if (j + 1 < T) release();   // V_j and K_j+1
                        if (j + 2 < T) {
                            const uint64_t desc_k = smem_desc(base + OFF_RING + take(false) * TILE, 16, 1024);
                            scores(t, desc_q, desc_k, 0, HD / 16);
                            if (elected) commit(bar(B_SFULL + t));
                        }
                        if (elected && (pass == 1 || j + 2 >= T)) commit(bar(B_PVDONE + t));
                    }
                    continue;
                }
                {
                    const uint64_t desc_k = smem_desc(base + OFF_RING + take(false) * TILE, 16, 1024);
                    for (int t = 0; t < n_tiles_q; ++t) {
                        mbar_wait_warp(bar(B_QFULL + t), (q_phase >> t) & 1, abort_flag, dev_status);
                        fence_after();
                        products_s(t, desc_k, 0, HD / 16);
                        if (elected) commit(bar(B_SFULL + t));
                    }
                    release();
                }
                bool kv_ready = false, p_ready = false;
                for (int j = 0; j < T; ++j) {
                    const bool more = j + 1 < T, more2 = j + 2 < T;
                    const int slot_v = take(kv_ready);
                    const uint64_t desc_v = smem_desc(base + OFF_RING + slot_v * TILE, SUB, 1024);
                    const uint64_t desc_k = smem_desc(base + OFF_RING + (more ? take(kv_ready) : 0) * TILE, 16, 1024);
                    if (j == j_end) zeroed(slot_v);
                    for (int t = 0; t < n_tiles_q; ++t) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (h == 1 || !p_ready) mbar_wait_warp(bar(B_PFULL + h * 2 + t), (p_phase >> t) & 1, abort_flag, dev_status);
                            fence_after();
                            outputs(t, desc_v, h, j > 0);
                        }
                        p_phase ^= 1u << t;
                        p_ready = false;
                        if (more) {
                            products_s(t, desc_k, 0, kPeek);
                            const int next = t + 1 == n_tiles_q ? 0 : t + 1;
                            const bool p_seen = mbar_test(bar(B_PFULL + next), (p_phase >> next) & 1);
                            if (t == 0) kv_ready = __all_sync(0xffffffffu, full(0) && (!more2 || full(1)));
                            p_ready = __all_sync(0xffffffffu, p_seen);
                            products_s(t, desc_k, kPeek, HD / 16);
                            if (elected) commit(bar(B_SFULL + t));
                        }
                        if (elected && (pass == 1 || !more)) commit(bar(B_PVDONE + t));
                    }
                    if (more) release();
                }
            }
            q_phase ^= n_tiles_q == 2 ? 3u : 1u;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_SEGFREE + it % kSegments));
        }
    } else {
        // ================================ softmax (warps 2..17) ================================
        uint32_t s_phase = 0, pv_phase = 0;   // of S, and by row tile of the finished products
        for (int it = 0;; ++it) {
            const Segment& seg = segments[it % kSegments];
            // one thread decides for these warps: named barriers know no time-out, so none of them may leave alone
            if (tid == 64) {
                mbar_wait(bar(B_SEGFULL + it % kSegments), (it / kSegments) & 1, abort_flag, dev_status);
                go[it & 1] = !*abort_flag && seg.more;
            }
            named_barrier(12, kSoftThreads);
            if (!uniform(go[it & 1])) break;
            const Job job(p.plan, seg);
            const int j0 = job.j0, T = job.T, kv = job.kv, rows = job.rows, n_chains = job.split ? 2 : job.n_tiles_q;
            const bool split = job.split;
            const int ws = warp - 2;
            const int t = ws >> 3, h = (ws >> 2) & 1;
            const int quarter = warp & 3;
            const int row = quarter * 32 + lane;
            const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
            const uint32_t tm_s = tmem + lane_addr + TM_S + t * 128;
            const uint32_t tm_o = tmem + lane_addr + TM_O + t * HD;
            float* xch_mine = xch + (t * 2 + h) * BM + row;
            const float* xch_other = xch + (t * 2 + (1 - h)) * BM + row;
            const int pair_bar = 1 + t * 4 + quarter;
            unsigned char* qtile = gbase + OFF_Q + t * TILE;
            auto piece = [&](int rw, int g) {   // 16-byte piece g of a row of the row tile: 128-byte swizzle
                return reinterpret_cast<uint4*>(qtile + (g >> 3) * SUB + (rw >> 3) * 1024 + (rw & 7) * 128 + (((g & 7) ^ (rw & 7)) << 4));
            };
            constexpr int RW = 32 / CH;   // rows at a time, CH lanes a half row
            const int sub = lane / CH, ch = lane % CH;
            if (t < n_chains) {
                const int tq = split ? 0 : t;              // row tile
                const int js = split ? 2 : 1;              // key tiles jt, jt + js, ...: nt of them
                const int jt = split ? t : 0, nt = (T - jt + js - 1) / js;
                int lim;   // keys that this row sees (rows behind the last: what the sequence has)
                {
                    const Places places(p.plan, seg.u);
                    // ---- Q: a warp its 32 rows, its half of the columns ----
                    if (tq == t) {
                        uint4 x[CH];
#pragma unroll
                        for (int k = 0; k < CH; ++k) {
                            const int r = t * BM + quarter * 32 + k * RW + sub;
                            x[k] = make_uint4(0, 0, 0, 0);
                            if (r < rows) x[k] = *reinterpret_cast<const uint4*>(p.q + places.element(r, p.n_q_heads, HD) + h * CW + ch * 8);
                        }
#pragma unroll
                        for (int k = 0; k < CH; ++k) *piece(quarter * 32 + k * RW + sub, h * CH + ch) = x[k];
                        fence_async_smem();
                        mbar_arrive(bar(B_QFULL + t));
                    }
                    const int r = tq * BM + row;
                    lim = r < rows ? limit_of(p.plan, seg.u.s, places.token(r)) : kv;
                }
                const int lim_low = __reduce_min_sync(0xffffffffu, lim);   // the fewest of the warp's rows
                float m_used = 0.f, l_run = 0.f;
                const float sl2 = p.scale_log2;
                const f32x2 sl2_2 = pk(sl2, sl2);
                {
                    f32x2 mneg2 = pk(0.f, 0.f), sum2[2] = {pk(0.f, 0.f), pk(0.f, 0.f)};
                    int key0 = (j0 + jt) * BN;   // of the tile
                    for (int i = 0; i < nt; ++i, key0 += js * BN) {
                        mbar_wait(bar(B_SFULL + t), s_phase, abort_flag, dev_status);
                        s_phase ^= 1;
                        fence_after();
                        if (i == 0) {
                            uint32_t r8[8];
                            ld8(tm_s, r8);
                            wait_ld<8>(r8);
                            // (a limit at or below the first key: the row sees nothing of this part)
                            if (lim > key0) {
                                float mx = __uint_as_float(r8[0]);
#pragma unroll
                                for (int c = 1; c < 8; ++c)
                                    if (key0 + c < lim) mx = fmaxf(mx, __uint_as_float(r8[c]));
                                m_used = mx * sl2;
                            }
                            mneg2 = pk(-m_used, -m_used);
                            named_barrier(pair_bar, 64);
                        }
                        uint32_t sr[2][32];
                        ld32(tm_s + h * 64, sr[0]);
                        wait_ld<32>(sr[0]);
                        ld32(tm_s + h * 64 + 32, sr[1]);
                        const bool masked = key0 + h * 64 + 64 > lim_low;
                        const int seen = lim - key0 - h * 64;   // columns of this half that the row sees
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (q == 1) wait_ld<32>(sr[1]);
                            if (masked) {
                                __syncwarp();   // (the same for the whole warp; without this the compiler makes 64 selects of every tile)
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (q * 32 + c >= seen) sr[q][c] = 0xff800000u;   // -inf
                            }
                            uint32_t pw[16];
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                const f32x2 d2 = fma2(pk(__uint_as_float(sr[q][2 * c]), __uint_as_float(sr[q][2 * c + 1])), sl2_2, mneg2);
                                float d0, d1;
                                upk(d2, d0, d1);
                                const float e0 = fast_exp2(d0), e1 = fast_exp2(d1);
                                sum2[c & 1] = add2(sum2[c & 1], pk(e0, e1));
                                pw[c] = pack_bf16x2(e0, e1);
                                if (q == 1 && c == 7) {
                                    st8(tm_s + h * 64 + 16, pw);
                                    wait_st();
                                    fence_before();
                                    mbar_arrive(bar(B_PFULL + t));
                                }
                            }
                            if (q == 0) {
                                st16(tm_s + h * 64, pw);
                            } else {
                                st8(tm_s + h * 64 + 24, pw + 8);
                                wait_st();
                                fence_before();
                                mbar_arrive(bar(B_PFULL + 2 + t));
                            }
                        }
                    }
                    float a0, a1, b0, b1;
                    upk(sum2[0], a0, a1);
                    upk(sum2[1], b0, b1);
                    l_run = (a0 + a1) + (b0 + b1);
                }
                const bool redo = named_barrier_or(n_chains == 2 ? 9 : 11, n_chains * 256, !(l_run <= kMaxSum));
                if (ws == 0 && lane == 0) {
                    again[it & 1] = redo ? 1 : 0;
                    mbar_arrive(bar(B_VERDICT));
                }
                // ---- second pass, only if a score left the first one's range: running maxima ----
                if (redo) {
                    m_used = -INFINITY;
                    l_run = 0.f;
                }
                // B_PVDONE: one phase at the end of the first pass, one per key tile of the second
                const uint32_t pv0 = (pv_phase >> t) & 1, last_phase = pv0 ^ (redo ? nt & 1 : 0);
                pv_phase ^= (redo ? (nt + 1) & 1 : 1) << t;
                for (int i = 0; redo && i < nt; ++i) {
                    mbar_wait(bar(B_SFULL + t), s_phase, abort_flag, dev_status);
                    s_phase ^= 1;
                    fence_after();
                    uint32_t sr[BN / 2];
                    ld32(tm_s + h * 64, sr);
                    ld32(tm_s + h * 64 + 32, sr + 32);
                    wait_ld<64>(sr);
                    const int key0 = (j0 + jt + i * js) * BN + h * 64;
                    if (key0 + 64 > lim_low) {
#pragma unroll
                        for (int c = 0; c < 64; ++c)
                            if (key0 + c >= lim) sr[c] = 0xff800000u;   // -inf
                    }
                    float mx[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) mx[c] = __uint_as_float(sr[c]);
#pragma unroll
                    for (int c = 4; c < 64; c += 2) mx[(c >> 1) & 3] = max3(mx[(c >> 1) & 3], __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]));
                    const float mloc = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    *xch_mine = mloc;
                    named_barrier(pair_bar, 64);
                    const float m_tile = fmaxf(mloc, *xch_other) * sl2;
                    float factor = 1.f;
                    if (m_tile > m_used + 8.f || (m_used == -INFINITY && m_tile > -INFINITY)) {   // stale maximum allowed up to 2^8
                        factor = (m_used == -INFINITY) ? 0.f : fast_exp2(m_used - m_tile);
                        m_used = m_tile;
                    }
                    const bool need_rescale = (i > 0) && __any_sync(0xffffffffu, factor != 1.f);
                    const float ref = m_used == -INFINITY ? 0.f : m_used;   // (a row that has seen nothing yet)
                    const f32x2 mneg2 = pk(-ref, -ref);
                    f32x2 sum2[2] = {pk(0.f, 0.f), pk(0.f, 0.f)};
                    uint32_t pw[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        const f32x2 d2 = fma2(pk(__uint_as_float(sr[2 * c]), __uint_as_float(sr[2 * c + 1])), sl2_2, mneg2);
                        float d0, d1;
                        upk(d2, d0, d1);
                        const float e0 = fast_exp2(d0), e1 = fast_exp2(d1);
                        sum2[c & 1] = add2(sum2[c & 1], pk(e0, e1));
                        pw[c] = pack_bf16x2(e0, e1);
                    }
                    {
                        float a0, a1, b0, b1;
                        upk(sum2[0], a0, a1);
                        upk(sum2[1], b0, b1);
                        l_run = fmaf(l_run, factor, (a0 + a1) + (b0 + b1));
                    }
                    if (need_rescale) {
                        mbar_wait(bar(B_PVDONE + t), pv0 ^ (i & 1), abort_flag, dev_status);
                        fence_after();
#pragma unroll
                        for (int c = 0; c < CW / 32; ++c) {
                            uint32_t o[32];
                            ld32(tm_o + h * CW + c * 32, o);
                            wait_ld<32>(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                            st32(tm_o + h * CW + c * 32, o);
                        }
                    }
                    st32(tm_s + h * 64, pw);
                    wait_st();
                    fence_before();
                    mbar_arrive(bar(B_PFULL + t));
                    mbar_arrive(bar(B_PFULL + 2 + t));
                }

                // ---- epilogue ------------------------------------------------------------------------
                mbar_wait(bar(B_PVDONE + t), last_phase, abort_flag, dev_status);
                fence_after();
                *xch_mine = l_run;
                named_barrier(pair_bar, 64);
                float l_row = l_run + *xch_other;
                float own = 1.f, odd = 0.f;   // weights of this chain's accumulator and, with split, of the odd tiles'
                if (split) {
                    named_barrier(pair_bar, 64);   // the halves' sums have been read
                    if (l_row == 0.f) m_used = -INFINITY;
                    if (h == 0) xch[t * 2 * BM + row] = m_used, xch[(t * 2 + 1) * BM + row] = l_row;   // (each chain in its own)
                    fence_before();
                    named_barrier(10, 512);        // (and every product is through, see the wait above)
                    fence_after();
                    const float m_odd = xch[2 * BM + row], l_odd = xch[3 * BM + row];
                    if (t == 0) {
                        const float M = fmaxf(m_used, m_odd), ref = M == -INFINITY ? 0.f : M;
                        own = fast_exp2(m_used - ref), odd = fast_exp2(m_odd - ref);
                        l_row = fmaf(own, l_row, odd * l_odd);
                        m_used = M;
                    }
                }
                // 32 columns of the row's output, un-normalised
                auto columns = [&](int c, uint32_t(&o)[32]) {
                    ld32(tm_o + h * CW + c * 32, o);
                    wait_ld<32>(o);
                    if (split) {
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            uint32_t x[16];
                            ld16(tm_o + HD + h * CW + c * 32 + part * 16, x);
                            wait_ld<16>(x);
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                o[part * 16 + e] = __float_as_uint(fmaf(own, __uint_as_float(o[part * 16 + e]), odd * __uint_as_float(x[e])));
                        }
                    }
                };
                const bool writes = tq == t;
                if (writes && j0 == 0 && T == seg.u.steps) {
                    // whole unit: normalised rows over the row tile's Q, and from there in pieces of 128 or 64 bytes to their places
                    const float inv = l_row > 0.f ? 1.f / l_row : 0.f;
#pragma unroll 1
                    for (int c = 0; c < CW / 32; ++c) {
                        uint32_t o[32];
                        columns(c, o);
#pragma unroll
                        for (int v4 = 0; v4 < 4; ++v4) {
                            uint4 w;
                            w.x = pack_bf16x2(__uint_as_float(o[v4 * 8 + 0]) * inv, __uint_as_float(o[v4 * 8 + 1]) * inv);
                            w.y = pack_bf16x2(__uint_as_float(o[v4 * 8 + 2]) * inv, __uint_as_float(o[v4 * 8 + 3]) * inv);
                            w.z = pack_bf16x2(__uint_as_float(o[v4 * 8 + 4]) * inv, __uint_as_float(o[v4 * 8 + 5]) * inv);
                            w.w = pack_bf16x2(__uint_as_float(o[v4 * 8 + 6]) * inv, __uint_as_float(o[v4 * 8 + 7]) * inv);
                            *piece(row, h * CH + c * 4 + v4) = w;
                        }
                    }
                    __syncwarp();
                    if (!*abort_flag) {   // a CTA whose wait gave up stores nothing
                        const Places places(p.plan, seg.u);
#pragma unroll
                        for (int k = 0; k < CH; ++k) {
                            const int rw = quarter * 32 + k * RW + sub, r = t * BM + rw;
                            const uint4 w = *piece(rw, h * CH + ch);
                            if (r < rows) *reinterpret_cast<uint4*>(p.out + places.element(r, p.n_q_heads, HD) + h * CW + ch * 8) = w;
                        }
                    }
                } else if (writes) {
                    // a part: un-normalised rows (relative to m_used), m and l
                    float* part = p.partial + ((long long)cta * 2 + (j0 == 0 ? 1 : 0)) * (2 * BM * (HD + 2));
                    if (t * BM + quarter * 32 < rows && !*abort_flag) {   // some of this warp's rows
                        float4* at = reinterpret_cast<float4*>(part) + ((t * (HD / 4) + h * (HD / 8)) * BM + row);
#pragma unroll 1
                        for (int c = 0; c < CW / 32; ++c) {
                            uint32_t o[32];
                            columns(c, o);
#pragma unroll
                            for (int v4 = 0; v4 < 8; ++v4)
                                at[(c * 8 + v4) * BM] = make_float4(__uint_as_float(o[v4 * 4]), __uint_as_float(o[v4 * 4 + 1]),
                                                                    __uint_as_float(o[v4 * 4 + 2]), __uint_as_float(o[v4 * 4 + 3]));
                        }
                        if (h == 0)   // (no weight on the reference of a row that saw nothing)
                            *reinterpret_cast<float2*>(part + 2 * BM * HD + (t * BM + row) * 2) = make_float2(l_row > 0.f ? m_used : -INFINITY, l_row);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_SEGFREE + it % kSegments));
        }
    }

    __syncthreads();
    if (warp == 1) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TM_COLS) : "memory");
    }
}

// the pool [n_pages, n_kv_heads, page_size, HD] seen as 4-D {64 columns, position, half, page and head}
bool make_page_map(CUtensorMap* map, const void* pool, const ec_paged_desc& d) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t row = (cuuint64_t)d.head_dim * 2, halves = (cuuint64_t)d.head_dim / 64;
    const cuuint64_t dims[4] = {64, (cuuint64_t)d.page_size, halves, (cuuint64_t)d.n_pages * d.n_kv_heads};
    const cuuint64_t strides[3] = {row, 128, row * d.page_size};
    const cuuint32_t box[4] = {64, (cuuint32_t)d.page_size, d.page_size == BN ? (cuuint32_t)halves : 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD>
cudaError_t launch(const PagedArgs& a, cudaStream_t stream) {
    CUtensorMap map_k, map_v;
    if (!make_page_map(&map_k, a.k_pages, a.d) || !make_page_map(&map_v, a.v_pages, a.d)) return cudaErrorInvalidValue;
    Params p;
    p.plan = make_plan(a, 2 * BM, BN);
    // (us, start 0 / 2 / 4 / 6 / 8 steps: chunks of 1100 to 1330 rows over up to 3750 keys 307 / 252 / 213 / 216 / 225; eight blocks
    // of up to 34 rows over up to 3540 keys with 32 heads 107 / 88 / 80 / 78 / 78)
    p.plan.start = 5;
    p.plan.min_steps = 2 + p.plan.start;
    p.q = static_cast<const __nv_bfloat16*>(a.q);
    p.out = static_cast<__nv_bfloat16*>(a.out);
    p.page_table = a.page_table;
    p.page_shift = __builtin_ctz((unsigned)a.d.page_size);
    p.n_pages = a.d.n_pages, p.max_pages = a.d.max_pages, p.n_q_heads = a.d.n_q_heads;
    p.scale_log2 = a.scale * kLog2e;
    const int ctas = sm_count();
    p.cuts = static_cast<Cut*>(a.workspace);
    p.partial = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + cuts_bytes(ctas));
    static PerDeviceOnce once;
    if (const cudaError_t e = ensure_dynamic_smem(once, attend_paged_tiles_kernel<HD>, (int)Geo<HD>::BYTES); e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = Geo<HD>::BYTES;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (const cudaError_t e = cudaLaunchKernelEx(&cfg, attend_paged_tiles_kernel<HD>, map_k, map_v, p); e != cudaSuccess) return e;
    return launch_combine<__nv_bfloat16, HD, true>(p.plan, p.cuts, p.partial, a.out, a.d.n_q_heads, ctas, stream);
}

}  // namespace

size_t attend_paged_tiles_workspace(const ec_paged_desc& d) {
    const int ctas = sm_count();
    return cuts_bytes(ctas) + (size_t)ctas * 2 * 2 * BM * (d.head_dim + 2) * 4;
}
// Up to sixteen packed rows the other kernel has less to do.  With more it takes the keys once for every sixteen, and is still
// the faster one while that is little: a unit of this kernel costs 8 us to start and end, and a few of them leave most SMs idle.
// (tile of 16 rows, kv head) pairs x room for keys (the lengths are not known here), us here / there: 46 k (8 x 300 rows of 300
// keys) 20.6 / 14.0; 48 k (2 x 40 of 1000, 8 heads) 26.9 / 14.8; 46 k (34 of 768, 28 heads on 4) 30.3 / 13.9; 131 k (4 x 8 of 2048, 32 on 8)
// 29.2 / 23.9; 262 k (20 of 4096, 32 heads) 33.6 / 29.5; 288 k (8 x 32 of 1500, 12 heads of 64) 27.1 / 29.6; 368 k (8 x 34 of 768, 28 on 4) 36.6 /
// 41.1; 786 k (34 of 8192, 32 heads) 44.5 / 54.9.
constexpr double kFewKeys = 270e3;
bool attend_paged_tiles_supported(const ec_paged_desc& d, int max_rows) {
    const long long rows = (long long)max_rows * (d.n_q_heads / d.n_kv_heads);
    if (d.dtype != EC_BF16 || rows <= 16 || (long long)d.n_pages * d.n_kv_heads > 0x7fffffffll) return false;
    return (double)((rows + 15) / 16) * d.batch * d.n_kv_heads * d.max_pages * d.page_size > kFewKeys;
}
cudaError_t launch_attend_paged_tiles(const PagedArgs& a, cudaStream_t stream) {
    return a.d.head_dim == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace ec
