// Page bookkeeping of the paged cache (ec_pages_fork / reserve / release / compact) and ec_pages_copy.
//
// The bookkeeping reads and writes a few kilobytes: what it costs is a launch and the dependent steps inside it, so each call
// is one CTA (release and the table pass of compact: a warp a sequence), and every order that a result depends on comes
// from a scan.  Atomics only count owners of a page, which no order changes.
// ec_pages_copy is bound by memory: every page is read once and written once, 16 bytes a lane, 16 KB of a CTA in flight:
// 940 MB 155 us, 6.0 TB/s.  fork 4.7 us, reserve 8.2, compact 9.9 + 6.7 (8320 pages, 64 sequences; behind one another less).
#include "ec_common.cuh"
#include "ec_tc_ptx.cuh"

namespace ec {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;

// Exclusive scan of one value a thread over the CTA; `total` for everybody.  Two barriers.
__device__ __forceinline__ int scan(int v, int& total, int* shared /* [kWarps + 1] */) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();   // the last scan's readers are through
    if (lane == 31) shared[warp] = x;
    __syncthreads();
    int below = 0, all = 0;
    int w = shared[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    below = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    all = __shfl_sync(0xffffffffu, w, 31);
    total = all;
    return (warp ? below : 0) + x - v;
}
__device__ __forceinline__ int pages_for(int len, int page_size) {   // (no sum: a page may be as long as an int)
    return len / page_size + (len % page_size != 0);
}
__device__ __forceinline__ int len_of(const ec_pages_desc& d, const int32_t* lens, int b) {
    return (int)min((long long)max(lens[b], 0), (long long)d.max_pages * d.page_size);
}

__global__ void __launch_bounds__(kThreads) fork_kernel(const ec_pages_desc d, int32_t* table, int32_t* lens, int32_t* refs,
                                                        const int32_t* src, const int32_t* dst, int n, int32_t* dev_status) {
    __shared__ int from[EC_PAGED_MAX_BATCH], to[EC_PAGED_MAX_BATCH], len[EC_PAGED_MAX_BATCH];
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    for (int i = threadIdx.x; i < n; i += kThreads) from[i] = src[i], to[i] = dst[i];
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int a = from[i], b = to[i];
        bool ok = a >= 0 && a < d.batch && b >= 0 && b < d.batch && lens[b] == 0;
        for (int j = 0; ok && j < i; ++j) ok = to[j] != b;
        len[i] = ok ? len_of(d, lens, a) : -1;
        if (!ok && dev_status) atomicExch(dev_status, (int)EC_ERR_SHAPE);
    }
    __syncthreads();   // every length has been read as it was
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = warp; i < n; i += kWarps) {
        if (len[i] < 0) continue;
        const int used = pages_for(len[i], d.page_size);
        const int32_t* a = table + (long long)from[i] * d.max_pages;
        int32_t* b = table + (long long)to[i] * d.max_pages;
        for (int e = lane; e < used; e += 32) {
            const int page = a[e];
            b[e] = page;
            if ((unsigned)page < (unsigned)d.n_pages) atomicAdd(refs + page, 1);
        }
        if (lane == 0 && from[i] != to[i]) lens[to[i]] = len[i];
    }
}

__global__ void __launch_bounds__(kThreads) reserve_kernel(const ec_pages_desc d, int32_t* table, int32_t* lens, int32_t* refs,
                                                           const int32_t* write_from, const int32_t* new_lens,
                                                           int32_t* copy_src, int32_t* copy_dst, int copy_cap,
                                                           int32_t* n_copies, int32_t* free_ids, int32_t* dev_status) {
    __shared__ int part[kWarps + 1];
    __shared__ int need[EC_PAGED_MAX_BATCH], copied[EC_PAGED_MAX_BATCH];   // of the sequences before this one, once scanned
    __shared__ int too_long;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) too_long = 0;
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    __syncthreads();
    // entries [first, have) that are shared are replaced, [have, want) are new
    auto range = [&](int b, int& first, int& have, int& upto, int& want) {
        const int len = len_of(d, lens, b), now = new_lens[b], from = max(write_from[b], 0);
        have = pages_for(len, d.page_size);
        want = max(have, pages_for(max(now, 0), d.page_size));
        upto = min(have, pages_for(max(now, 0), d.page_size));
        first = from < now ? from / d.page_size : upto;
    };
    for (int b = warp; b < d.batch; b += kWarps) {
        int first, have, upto, want;
        if ((long long)new_lens[b] > (long long)d.max_pages * d.page_size) {
            if (lane == 0) too_long = 1, need[b] = copied[b] = 0;
            continue;
        }
        range(b, first, have, upto, want);
        int c = 0;
        for (int e = first + lane; e < upto; e += 32) {
            const int page = table[(long long)b * d.max_pages + e];
            c += (unsigned)page < (unsigned)d.n_pages && refs[page] > 1;
        }
        c = __reduce_add_sync(0xffffffffu, c);
        if (lane == 0) need[b] = c + want - have, copied[b] = c;
    }
    __syncthreads();
    int all_need, all_copied;
    const int mine = tid < d.batch ? need[tid] : 0, mine_c = tid < d.batch ? copied[tid] : 0;
    const int before = scan(mine, all_need, part), before_c = scan(mine_c, all_copied, part);
    __syncthreads();
    if (tid < d.batch) need[tid] = before, copied[tid] = before_c;
    // the lowest free ids, as many as are needed
    int found = 0;
    for (int p0 = 0; p0 < d.n_pages && found < all_need; p0 += 4 * kThreads) {
        const int p = p0 + 4 * tid;
        bool f[4];
        int c = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = p + i < d.n_pages && refs[p + i] == 0;
            c += f[i];
        }
        int total;
        int at = found + scan(c, total, part);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (f[i]) free_ids[at++] = p + i;
        found += total;
    }
    __syncthreads();
    const bool ok = !too_long && found >= all_need && all_copied <= copy_cap;
    const int pairs = ok ? all_copied : 0;
    for (int i = pairs + tid; i < copy_cap; i += kThreads) copy_src[i] = copy_dst[i] = -1;
    if (tid == 0) {
        *n_copies = pairs;
        if (!ok && dev_status) atomicExch(dev_status, (int)EC_ERR_PAGE);
    }
    if (!ok) return;
    for (int b = warp; b < d.batch; b += kWarps) {
        int first, have, upto, want;
        range(b, first, have, upto, want);
        int32_t* row = table + (long long)b * d.max_pages;
        int at = need[b], at_c = copied[b];
        for (int e0 = first; e0 < upto; e0 += 32) {
            const int e = e0 + lane, page = e < upto ? row[e] : -1;
            const bool shared = (unsigned)page < (unsigned)d.n_pages && refs[page] > 1;
            const uint32_t m = __ballot_sync(0xffffffffu, shared);
            if (shared) {
                const int k = __popc(m & ((1u << lane) - 1u)), id = free_ids[at + k];
                row[e] = id;
                copy_src[at_c + k] = page;
                copy_dst[at_c + k] = id;
            }
            at += __popc(m);
            at_c += __popc(m);
        }
        for (int e = have + lane; e < want; e += 32) row[e] = free_ids[at + e - have];
        __syncwarp();
        if (lane == 0) lens[b] = max(len_of(d, lens, b), new_lens[b]);
    }
    __syncthreads();   // every decision has been made on the counts as they were
    for (int i = tid; i < all_need; i += kThreads) refs[free_ids[i]] = 1;
    for (int i = tid; i < pairs; i += kThreads) atomicSub(refs + copy_src[i], 1);
}

__global__ void __launch_bounds__(128) release_kernel(const ec_pages_desc d, int32_t* table, int32_t* lens, int32_t* refs,
                                                      const int32_t* keep_lens) {
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (b >= d.batch) return;
    const int len = len_of(d, lens, b), keep = max(keep_lens[b], 0);
    if (keep >= len) return;
    const int last = pages_for(len, d.page_size);
    for (int e = pages_for(keep, d.page_size) + lane; e < last; e += 32) {
        int32_t* entry = table + (long long)b * d.max_pages + e;
        const int page = *entry;
        if ((unsigned)page < (unsigned)d.n_pages) atomicSub(refs + page, 1);
        *entry = -1;
    }
    __syncwarp();
    if (lane == 0) lens[b] = keep;
}

// to[page]: where a page goes, -1 where it stays
__global__ void __launch_bounds__(kThreads) compact_plan_kernel(const ec_pages_desc d, int32_t* refs, int32_t* copy_src,
                                                                int32_t* copy_dst, int copy_cap, int32_t* n_copies, int32_t* to) {
    __shared__ int part[kWarps + 1];
    const int tid = threadIdx.x;
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    int mine = 0;
    for (int p = tid; p < d.n_pages; p += kThreads) {
        mine += refs[p] > 0;
        to[p] = -1;
    }
    int used;
    scan(mine, used, part);
    // i-th free id below `used` and i-th id in use from there on: equally many
    int n_dst = 0, n_src = 0;
    for (int p0 = 0; p0 < d.n_pages; p0 += 4 * kThreads) {
        const int p = p0 + 4 * tid;
        bool hole[4], move[4];
        int c = 0;   // holes in the low half, moves in the high half: at most 4096 each
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = p + i < d.n_pages, live = in && refs[p + i] > 0;
            hole[i] = in && !live && p + i < used;
            move[i] = live && p + i >= used;
            c += hole[i] + (move[i] << 16);
        }
        int total;
        const int at = scan(c, total, part);
        int ah = n_dst + (at & 0xffff), am = n_src + (at >> 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (hole[i] && ah < copy_cap) copy_dst[ah] = p + i;
            if (move[i] && am < copy_cap) copy_src[am] = p + i;
            ah += hole[i];
            am += move[i];
        }
        n_dst += total & 0xffff;
        n_src += total >> 16;
    }
    __syncthreads();
    const int n = min(n_src, copy_cap);
    for (int i = tid; i < n; i += kThreads) {
        const int a = copy_src[i], b = copy_dst[i];
        to[a] = b;
        refs[b] = refs[a];
        refs[a] = 0;
    }
    for (int i = n + tid; i < copy_cap; i += kThreads) copy_src[i] = copy_dst[i] = -1;
    if (tid == 0) *n_copies = n;
}
__global__ void __launch_bounds__(128) compact_table_kernel(const ec_pages_desc d, int32_t* table, const int32_t* lens,
                                                            const int32_t* to) {
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (b >= d.batch) return;
    const int used = pages_for(len_of(d, lens, b), d.page_size);
    for (int e = lane; e < used; e += 32) {
        int32_t* entry = table + (long long)b * d.max_pages + e;
        const int page = *entry;
        if ((unsigned)page < (unsigned)d.n_pages && to[page] >= 0) *entry = to[page];
    }
}

constexpr int kCopyThreads = 256, kCopyChunk = kCopyThreads * 64;   // bytes
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(unsigned char* k, unsigned char* v, long long page_bytes, int n_pages,
                                                            int n_layers, long long layer_bytes, const int32_t* src,
                                                            const int32_t* dst, int cap, const int32_t* n_copies,
                                                            int32_t* dev_status) {
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    const int n = n_copies ? min(max(*n_copies, 0), cap) : cap;
    const int per = (int)((page_bytes + kCopyChunk - 1) / kCopyChunk);   // chunks of a page
    const long long items = (long long)n * n_layers * 2 * per;
    for (long long i = blockIdx.x; i < items; i += gridDim.x) {
        const int chunk = (int)(i % per);
        const long long rest = i / per;
        const int which = (int)(rest & 1), layer = (int)((rest >> 1) % n_layers);
        const int pair = (int)((rest >> 1) / n_layers);
        const int a = src[pair], b = dst[pair];
        if ((unsigned)a >= (unsigned)n_pages || (unsigned)b >= (unsigned)n_pages) {
            if (threadIdx.x == 0 && dev_status) atomicExch(dev_status, (int)EC_ERR_PAGE);
            continue;
        }
        unsigned char* pool = (which ? v : k) + layer * layer_bytes;
        const long long at = (long long)chunk * kCopyChunk + threadIdx.x * 16;
        const uint4* from = reinterpret_cast<const uint4*>(pool + a * page_bytes + at);
        uint4* to = reinterpret_cast<uint4*>(pool + b * page_bytes + at);
        uint4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (at + j * kCopyThreads * 16 < page_bytes) x[j] = __ldcs(from + j * kCopyThreads);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (at + j * kCopyThreads * 16 < page_bytes) to[j * kCopyThreads] = x[j];
    }
}

template <typename... P, typename... A>
cudaError_t run(void (*kernel)(P...), int grid, int block, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(block, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace

cudaError_t launch_pages_fork(const ec_pages_desc& d, int32_t* table, int32_t* lens, int32_t* refs, const int32_t* src,
                              const int32_t* dst, int n, int32_t* dev_status, cudaStream_t stream) {
    return run(fork_kernel, 1, kThreads, stream, d, table, lens, refs, src, dst, n, dev_status);
}
cudaError_t launch_pages_reserve(const ec_pages_desc& d, int32_t* table, int32_t* lens, int32_t* refs,
                                 const int32_t* write_from, const int32_t* new_lens, int32_t* copy_src, int32_t* copy_dst,
                                 int copy_cap, int32_t* n_copies, void* workspace, int32_t* dev_status, cudaStream_t stream) {
    return run(reserve_kernel, 1, kThreads, stream, d, table, lens, refs, write_from, new_lens, copy_src, copy_dst, copy_cap,
               n_copies, static_cast<int32_t*>(workspace), dev_status);
}
cudaError_t launch_pages_release(const ec_pages_desc& d, int32_t* table, int32_t* lens, int32_t* refs,
                                 const int32_t* keep_lens, cudaStream_t stream) {
    return run(release_kernel, (d.batch + 3) / 4, 128, stream, d, table, lens, refs, keep_lens);
}
size_t pages_workspace_bytes(int n_pages) { return ((size_t)n_pages * 4 + 15) & ~(size_t)15; }
cudaError_t launch_pages_compact(const ec_pages_desc& d, int32_t* table, const int32_t* lens, int32_t* refs, int32_t* copy_src,
                                 int32_t* copy_dst, int copy_cap, int32_t* n_copies, void* workspace, cudaStream_t stream) {
    int32_t* to = static_cast<int32_t*>(workspace);
    if (const cudaError_t e = run(compact_plan_kernel, 1, kThreads, stream, d, refs, copy_src, copy_dst, copy_cap, n_copies, to);
        e != cudaSuccess)
        return e;
    return run(compact_table_kernel, (d.batch + 3) / 4, 128, stream, d, table, lens, to);
}
cudaError_t launch_pages_copy(void* k_pages, void* v_pages, long long page_bytes, int n_pages, int n_layers,
                              long long layer_bytes, const int32_t* src, const int32_t* dst, int cap,
                              const int32_t* n_copies, int32_t* dev_status, cudaStream_t stream) {
    const long long chunks = (long long)cap * n_layers * 2 * ((page_bytes + kCopyChunk - 1) / kCopyChunk);
    const long long most = (long long)sm_count() * 8;
    return run(copy_kernel, (int)(chunks < most ? chunks : most), kCopyThreads, stream, static_cast<unsigned char*>(k_pages),
               static_cast<unsigned char*>(v_pages), page_bytes, n_pages, n_layers, layer_bytes, src, dst, cap, n_copies, dev_status);
}

}  // namespace ec
