// ec_sample: one token per logits row from temperature, top-k, top-p, min-p and a given uniform number.
//
// With the tokens ordered by (logit, descending; index, ascending) every filter keeps a prefix, so a row is three searches
// for a rank: the k-th token (by count), the one at which the weights reach top_p of the sum so far (by weight), and the
// one at which they exceed u of the kept sum (by weight).  Nothing sorts the row.  In the order of the code:
//   1  the row's largest and smallest logit; the row's segments go to shared memory on the way where they fit;
//   2  by_estimate(): counts of 1024 fine bins say where the three places are, to within a few bins; one pass forms the
//      weights, sums those in front of each place exactly and takes the tokens around it; one CTA settles the rest
//      among these few thousand.  Rows with a top k whose prefix fits the list weigh nothing but that prefix;
//   3  where equal logits (a constant row) or an estimate that was off leave that undone, weights by 16 bins and searches that
//      narrow one bin down, at worst to single tokens: a few rows in a thousand, and some 80 us each.
//
// Weights are exp of fp64 arguments, rounded once to units of 2^-47 to 2^-43 of the largest weight (by the vocabulary alone,
// see unit_bits_of) and summed as integers.  fp32 sums of 10^5 weights would be off by some 10^-7 of their total, as much as a
// small weight itself: the token found would depend on the order of the sum.  Integers also make results independent of
// how many CTAs share a row.
//
// A row is shared by a cluster of 1 to 8 CTAs, each with a contiguous segment of it.  In step 3 a thread has a column of its own
// in the bins (16 x 512 x 8 bytes, no atomics, no bank conflicts): weight sum in the low 53 bits, count in the top 11.
//
// Bound by instructions: some 45 a token for a weight (ten of them 64-bit).  256 x 152064 in bf16, two CTAs a row: 58 % of the issue
// slots of an SM while it works, 28 % over the launch, which the slowest rows end; the bytes 4 % of the peak.  Of a row without top k on four CTAs (126464 tokens in fp32, clocks): step 1 13 k, counts and places 12 k, weights and
// taking 20 to 22 k, settling 11 to 20 k; with a top k of 200 48 k in all.  32 rows 37 to 43 us, 256 of 152064 in bf16 197 to 300
// (both by the rows).
#include "ec_common.cuh"
#include "ec_tc_ptx.cuh"

#include <cooperative_groups.h>

#include <cmath>
#include <type_traits>

namespace ec {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 16, kZeroBin = kBins - 1;   // the last: weights that round to 0
constexpr int kBinBits = 4;
static_assert(1 << kBinBits == kBins, "bins");
constexpr int kWeightBits = 53;            // of a thread's column of a bin; the rest counts
constexpr int kMaxCluster = 8;
constexpr int kSegment = kThreads * 1016;  // tokens of a CTA: 1016 weights of 2^43 units fit a thread's column
constexpr int kList = kThreads * kBins / 2;   // candidates that a search takes out of the row: two lists of them over the bins
constexpr int kFew = 128;                  // candidates that are ranked against one another
constexpr uint32_t HIST_BYTES = kBins * kThreads * 8;
constexpr int kMaxDynamic = 232448 - 34816;   // (the rest: struct Shared)
constexpr int kMaxUnitBits = 47;
// a thread's weights, none above one, have to stay below 2^kWeightBits: as fine a unit as the whole row on one CTA leaves room for
__host__ __device__ constexpr int unit_bits_of(int vocab) {
    int bits = kMaxUnitBits;
    while (bits > 43 && (long long)((vocab + 4095) / 4096 * 8) << bits >= 1ll << kWeightBits) --bits;
    return bits;
}
constexpr int kFine = 1024;                // fine bins: counts alone; the last: weights that round to 0
typedef unsigned long long u64;

// 2^(i / 64), i = 0 .. 63, from its definition; a copy for each of sixteen lanes (a half warp's 8-byte loads never meet in a bank)
struct ExpTable {
    double v[64][16];
};

// Order of a logit as an integer, ascending with DESCENDING logits; both zeros alike
__device__ __forceinline__ uint32_t order_of(float x) {
    uint32_t b = __float_as_uint(x);
    if (b == 0x80000000u) b = 0;
    return (b & 0x80000000u) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float((o & 0x80000000u) ? o : (~o & 0x7fffffffu));
}

// shared memory by its own addresses
__device__ __forceinline__ u64 lds64(uint32_t at) {
    u64 v;
    asm volatile("ld.shared.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts64(uint32_t at, u64 v) { asm volatile("st.shared.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t at, const uint4& v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

struct Scale {   // what turns a logit of this row into a bin and a weight
    float top, per_bin;   // bin = (top - x) * per_bin, to the nearest
    float low;            // what is below it weighs nothing
    float per_fine, nats;   // the same for the fine bins, and what a fine bin spans
    double wide_top, c;   // (x - top) * c = 64 log2 of the weight
    uint32_t table;       // shared address of this lane's copy of ExpTable
    double round, unit;   // 2^(52 - bits), whose last bit is one unit of weight, and 2^bits
};
// (every step of these three is monotone in x, so what they tell apart are intervals of the order)
__device__ __forceinline__ float depth_of(const Scale& s, float x) { return fminf((s.top - x) * s.per_bin, (float)kZeroBin); }
__device__ __forceinline__ int bin_of(const Scale& s, float x) { return __float_as_int(depth_of(s, x) + 8388608.f) & kZeroBin; }
__device__ __forceinline__ int fine_of(const Scale& s, float x) {
    return __float_as_int(fminf((s.top - x) * s.per_fine, (float)(kFine - 1)) + 8388608.f) & (kFine - 1);
}
// part of the interval [z0, z0 + parts / per_part) of depths
__device__ __forceinline__ int part_of(const Scale& s, float x, float z0, float per_part, int parts) {
    return min(max(__float2int_rz((depth_of(s, x) - z0) * per_part), 0), parts - 1);
}
// sum over the warp, exact while it fits
__device__ __forceinline__ u64 warp_sum(u64 v) {
    const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)(v & 0x3ffffffu)), b = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 26) & 0x3ffffffu),
                   c = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 52));
    return a + ((u64)b << 26) + ((u64)c << 52);
}
__device__ __forceinline__ u64 warp_min(u64 v) {
    const uint32_t h = __reduce_min_sync(0xffffffffu, (uint32_t)(v >> 32));
    return (u64)h << 32 | __reduce_min_sync(0xffffffffu, (uint32_t)(v >> 32) == h ? (uint32_t)v : 0xffffffffu);
}
__device__ __forceinline__ u64 warp_max(u64 v) { return ~warp_min(~v); }
// Weight in (0, 1], relative error 1e-13: 2^(n/64) from the table, 2^(r/64) for |r| <= 1/2 by its Taylor polynomial
// ((ln 2 / 128)^5 / 120 = 4e-14 left).  (x - top) * c must be above -64 * 60.
struct Parts {
    double poly, scale;
};
__device__ __forceinline__ Parts weight_parts(const Scale& s, float x) {
    constexpr double kMagic = 6755399441055744.0;   // 1.5 * 2^52: the sum's low bits are the nearest integer
    constexpr double a1 = 0.010830424696249145, a2 = a1 * a1 / 2, a3 = a1 * a1 * a1 / 6, a4 = a1 * a1 * a1 * a1 / 24;   // ln 2 / 64
    const double u = ((double)(x) - s.wide_top) * s.c;
    const double km = u + kMagic;
    const int k = __double2loint(km);
    const double r = u - (km - kMagic);
    const double p = fma(fma(fma(fma(a4, r, a3), r, a2), r, a1), r, 1.0);
    double t;   // (not volatile: the table stays as it is)
    asm("ld.shared.f64 %0, [%1];" : "=d"(t) : "r"(s.table + (k & 63) * 128));
    return {p, __hiloint2double(__double2hiint(t) + (k >> 6) * (1 << 20), __double2loint(t))};
}
// units of weight + bits(s.round)
__device__ __forceinline__ u64 weight_raw(const Scale& s, float x) {
    const Parts w = weight_parts(s, x);
    return (u64)__double_as_longlong(fma(w.poly, w.scale, s.round));
}
__device__ __forceinline__ u64 weight_units(const Scale& s, float x) {
    return weight_raw(s, x) - (u64)__double_as_longlong(s.round);
}

struct Found {    // the token that a search ends at
    u64 count, weight;   // of the tokens up to it, itself included
    u64 order;           // order << 32 | index
};

struct Shared {
    ExpTable tab;
    u64 xch[2][kMaxCluster][72];   // exchanged between the CTAs of a row: per rank 32 weights, 32 counts, 8 more
    u64 bin_w[kBins], bin_c[kBins], all_w, all_c, red_a[kWarps], red_b[kWarps];
    Found found;
    u64 cand_w[kFew];
    u64 part_w[256];
    uint32_t part_c[256];
    uint32_t fine[kFine], cum_c[kFine];   // counts of this CTA; of the row, running
    float cum_e[kFine];                   // running weights, estimated from the counts
    int done;
    uint32_t n_list, n_next;
    u64 pick[4];
};

// 8 consecutive logits as loaded, -inf past `end`
__device__ __forceinline__ void unpack8(const uint4 (&raw)[1], int i, int end, float (&x)[8]) {
    const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
    }
    if (i + 8 > end) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j >= end) x[j] = -INFINITY;
    }
}
__device__ __forceinline__ void unpack8(const uint4 (&raw)[2], int i, int end, float (&x)[8]) {
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
    if (i + 8 > end) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j >= end) x[j] = -INFINITY;
    }
}
// 8 consecutive logits, -inf past `end`
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int i, int end, float (&x)[8]) {
    uint4 v = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    if (i < end) v = *reinterpret_cast<const uint4*>(row + i);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
    if (i + 8 > end) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j >= end) x[j] = -INFINITY;
    }
}
__device__ __forceinline__ void load8(const float* row, int i, int end, float (&x)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (i + 4 * h < end) v = *reinterpret_cast<const float4*>(row + i + 4 * h);
        x[4 * h] = v.x, x[4 * h + 1] = v.y, x[4 * h + 2] = v.z, x[4 * h + 3] = v.w;
    }
    if (i + 8 > end) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j >= end) x[j] = -INFINITY;
    }
}

static_assert(sizeof(Shared) + kMaxDynamic <= 232448, "shared memory");

template <typename T, bool kResident>
class RowSampler {
public:
    __device__ RowSampler(Shared& sh, unsigned char* hist, uint32_t kept, const T* row, int begin, int end)
        : sh(sh), hist(hist), kept(kept), row(row), begin(begin), end(end), cluster(cg::this_cluster()), rank(cluster.block_rank()),
          n_ranks(cluster.num_blocks()), tid(threadIdx.x), lane(threadIdx.x & 31), warp(threadIdx.x >> 5) {}

    __device__ void run(const SampleArgs& a, int r) {
        // ---- largest logit (lowest index on ties) and the smallest finite one ----
        u64 best = ~0ull;
        uint32_t low = 0;
        first_pass([&](float x, int i) {
            if (x > -INFINITY) {
                const uint32_t o = order_of(x);
                best = min(best, (u64)o << 32 | (uint32_t)i);
                low = max(low, o);
            }
        });
        u64 low64 = low;
        block_min_max(best, low64);
        tc::cluster_wait();   // (the row's other CTAs have started: their shared memory may be written)
        publish(64, best), publish(65, low64);
        const u64(*in)[72] = exchange();
        best = ~0ull, low64 = 0;
        for (int k = 0; k < n_ranks; ++k) best = min(best, in[k][64]), low64 = max(low64, in[k][65]);
        float t = a.temperature ? a.temperature[r] : 1.f;
        // (beside an infinite logit no other one weighs anything)
        if (best == ~0ull || !(t > 0.f) || (uint32_t)(best >> 32) == order_of(INFINITY)) {
            if (rank == 0 && tid == 0) {
                const bool some = best != ~0ull;
                a.token_out[r] = some ? (int)(uint32_t)best : -1;
                if (a.prob_out) a.prob_out[r] = some ? 1.f : 0.f;
                if (a.kept_out) a.kept_out[r] = some ? 1 : 0;
            }
            return;
        }
        // (Below 2^-126 it counts as that: per_bin and per_fine are finite, so a row of logits within 10^-36 of one another stays in
        // the first bins however far a smaller t spreads its weights, and their exponents, over 2^1022, would wrap.)
        t = fmaxf(t, 1.17549435e-38f);
        s.top = value_of((uint32_t)(best >> 32));
        s.c = 64.0 * 1.4426950408889634074 / (double)t;
        s.table = tc::s2u(&sh.tab.v[0][tid & 15]);
        s.wide_top = (double)(s.top);
        const int bits = unit_bits_of(a.vocab);
        s.round = (double)(1ull << (52 - bits)), s.unit = (double)(1ull << bits);
        // the other bins over the nats above half a unit, (bits + 1) ln 2 < 33.4 of them, or over the whole row where that spans less
        const float span = (s.top - value_of((uint32_t)low64)) / t;
        s.per_bin = fminf((kZeroBin - 0.55f) / fmaxf(fminf(span * 1.001f, 33.4f), 1e-30f) / t, 1e37f);   // (finite: 0 times it is 0)
        s.nats = fmaxf(fminf(span * 1.001f, 33.4f), 1e-30f) / (kFine - 1.6f);
        s.per_fine = fminf(1.f / s.nats / t, 1e37f);
        s.low = s.top - kZeroBin / s.per_bin;
        const int k = a.top_k ? a.top_k[r] : 0;
        const float p = a.top_p ? a.top_p[r] : 1.f;
        const double u = (double)a.u[r];
        const float mp = a.min_p ? a.min_p[r] : 0.f;
        // What min-p keeps, as a bound of the logit: w >= min_p where x >= top + t ln(min_p), formed in 64 bits (weights in units
        // would tell min_p = 1e-13 apart to 4 %).  The 2^-54 stands for weights that are 1 in 64 bits.  The largest always stays.
        const float least = mp > 0.f ? __double2float_ru(s.wide_top + (double)t * (log((double)mp) - 5.6e-17)) : 0.f;
        constexpr u64 kOne = 1ull << kWeightBits;
        if (by_estimate(a, r, k, p, mp, u, least)) return;

        // ---- what the estimates could not settle: weights by bin, and searches that narrow a bin down ----
        const uint32_t column = tc::s2u(hist) + tid * 8;
#pragma unroll
        for (int b = 0; b < kBins; ++b) sts64(column + b * (kThreads * 8), 0);
        u64 kept_c = 0, kept_w = 0;
        // (eight weights at a time without a branch: one alone is a chain of ten 64-bit operations)
        const auto weigh = [&](auto with_floor) {
            const u64 one = kOne - (u64)__double_as_longlong(s.round);
            each8([&](const float(&x)[8], int) {
                u64 w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = weight_raw(s, fmaxf(x[j], s.low));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int b = bin_of(s, x[j]);
                    u64 add = w[j] + one;
                    if (b == kZeroBin) add = x[j] > -INFINITY ? kOne : 0;
                    bump(column, b, add);
                    if constexpr (decltype(with_floor)::value) {
                        const u64 units = add & (kOne - 1);
                        const bool in = add && x[j] >= least;
                        kept_c += in, kept_w += in ? units : 0;
                    }
                }
            });
        };
        if (mp > 0.f) weigh(std::true_type{});
        else weigh(std::false_type{});
        block_sum(kept_c, kept_w);
        reduce_bins();
        publish(64, kept_c), publish(65, kept_w);
        const u64(*all)[72] = exchange();
        sum_bins(all);
        kept_c = kept_w = 0;
        for (int k = 0; k < n_ranks; ++k) kept_c += all[k][64], kept_w += all[k][65];
        __syncthreads();

        // ---- the kept prefix, then the token in it ----
        u64 n = sh.all_c, sum = sh.all_w;
        if (k > 0 && (u64)k < n) {
            const Found f = search(true, k);
            n = k, sum = f.weight;
        }
        if (p < 1.f) {
            const Found f = search(false, reach(p, sum));
            if (f.count < n) n = f.count, sum = f.weight;
        }
        if (mp > 1.f) kept_c = 1, kept_w = (u64)s.unit;   // nobody reaches it: the first token alone
        if (mp > 0.f && kept_c < n) n = kept_c, sum = kept_w;
        answer(a, r, search(false, pass(u, sum)), n, sum);
    }

private:
    Shared& sh;
    unsigned char* hist;
    const uint32_t kept;   // the segment in shared memory
    const T* const row;
    const int begin, end;
    cg::cluster_group cluster;
    const int rank, n_ranks, tid, lane, warp;
    Scale s;
    int turn = 0;

    static __device__ __forceinline__ void bump(uint32_t column, int b, u64 add) {
        const uint32_t at = column + b * (kThreads * 8);
        sts64(at, lds64(at) + add);
    }
    // the first running sums that reach p of `sum`, and that exceed u of it
    static __device__ __forceinline__ u64 reach(float p, u64 sum) { return min((u64)fmax(1.0, ceil((double)p * (double)sum)), sum); }
    static __device__ __forceinline__ u64 pass(double u, u64 sum) { return min((u64)fmax(0.0, u * (double)sum) + 1, sum); }
    __device__ __forceinline__ void answer(const SampleArgs& a, int r, const Found& f, u64 n, u64 sum) {
        if (rank != 0 || tid != 0) return;
        a.token_out[r] = (int)(uint32_t)f.order;
        if (a.prob_out) {
            const Parts w = weight_parts(s, value_of((uint32_t)(f.order >> 32)));
            a.prob_out[r] = (float)(w.poly * w.scale * s.unit / (double)sum);
        }
        if (a.kept_out) a.kept_out[r] = (int)n;
    }
    __device__ __forceinline__ void sum_bins(const u64 (*all)[72]) {
        if (tid >= 32) return;
        u64 w = 0, c = 0;
        for (int k = 0; k < n_ranks && tid < kBins; ++k) w += all[k][tid], c += all[k][32 + tid];
        const u64 tw = warp_sum(w), tc = warp_sum(c);
        if (tid < kBins) sh.bin_w[tid] = w, sh.bin_c[tid] = c;
        if (tid == 0) sh.all_w = tw, sh.all_c = tc;
    }
    // ---- by estimate ----
    // Counts of 1024 fine bins (one 32-bit addition in shared memory a token, 11 a clock; weights would be 64-bit ones, of
    // which there are 1.4) give the place of the k-th token exactly, and, times the weight at a bin's middle, the places where
    // the running weight reaches what top-p and u ask for to within a fraction of a bin.  One more pass then forms all weights,
    // sums those in front of each place and takes the tokens of the bins around it; rank 0 finds the tokens among these, and sees
    // from the exact sums whether they stand there.  Where a top k is given and all tokens up to the k-th fit the list, it takes
    // them all, and no other weight is formed.
    struct Place {
        int lo, hi;   // fine bins; lo > hi: not asked for
    };
    // First fine bin at which the running value, no longer below `target`, is; whole warps, two loads
    template <typename V>
    __device__ __forceinline__ int bin_reaching(const V* cum, V target) const {
        const int block = min(__popc(__ballot_sync(0xffffffffu, cum[lane * 32 + 31] < target)), 31);
        return block * 32 + min(__popc(__ballot_sync(0xffffffffu, cum[block * 32 + lane] < target)), 31);
    }
    __device__ __forceinline__ int bin_of_count(uint32_t target) const { return bin_reaching<uint32_t>(sh.cum_c, target); }
    __device__ __forceinline__ int bin_of_estimate(float v) const { return min(bin_reaching<float>(sh.cum_e, v), kFine - 2); }
    // Around the place where the running weight is `v`.  A bin's estimate is off by a factor of e^(nats / 2) at most, and so is
    // every running one: `sure`.  Over many tokens the errors cancel, and a tenth of a bin nearly always holds the place: `narrow`,
    // one bin or two (a few hundred tokens of a flat row, whose taking costs); where it does not, a quarter and a bin to either side.
    enum Width { narrow, usual, sure };
    __device__ __forceinline__ Place around(float v, int width) const {
        const float margin = (width == sure ? 0.55f : width == usual ? 0.25f : 0.1f) * s.nats + 2e-5f;
        const int more = width == narrow ? 0 : 1;
        return Place{max(bin_of_estimate(v * (1.f - margin)) - more, 0), min(bin_of_estimate(v * (1.f + margin)) + more, kFine - 2)};
    }
    __device__ bool by_estimate(const SampleArgs& a, int r, int k, float p, float mp, double u, float least) {
        for (int i = tid; i < kFine; i += kThreads) sh.fine[i] = 0;
        __syncthreads();
        each8([&](const float(&x)[8], int) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (x[j] > -INFINITY) atomicAdd(&sh.fine[fine_of(s, x[j])], 1u);
        });
        cluster.sync();
        {   // running counts and estimates, two bins a thread
            static_assert(kFine == 2 * kThreads, "two fine bins a thread");
            uint32_t c0 = 0, c1 = 0;
            for (int q = 0; q < n_ranks; ++q) {
                const uint2 v = reinterpret_cast<const uint2*>(cluster.map_shared_rank(sh.fine, q))[tid];
                c0 += v.x, c1 += v.y;
            }
            const float l2 = -1.4426950f * s.nats;
            const float e0 = c0 * exp2f(l2 * (2 * tid)), e1 = tid == kThreads - 1 ? 0.f : c1 * exp2f(l2 * (2 * tid + 1));
            uint32_t pc = c0 + c1;
            float pe = e0 + e1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t xc = __shfl_up_sync(0xffffffffu, pc, o);
                const float xe = __shfl_up_sync(0xffffffffu, pe, o);
                if (lane >= o) pc += xc, pe += xe;
            }
            __syncthreads();
            if (lane == 31) sh.red_a[warp] = pc, sh.red_b[warp] = __float_as_uint(pe);
            __syncthreads();
            for (int q = 0; q < warp; ++q) pc += (uint32_t)sh.red_a[q], pe += __uint_as_float((uint32_t)sh.red_b[q]);
            sh.cum_c[2 * tid] = pc - c1, sh.cum_c[2 * tid + 1] = pc;
            sh.cum_e[2 * tid] = pe - e1, sh.cum_e[2 * tid + 1] = pe;
            __syncthreads();
        }
        // ---- the places ----
        const uint32_t live = sh.cum_c[kFine - 1];
        const bool cut_k = k > 0 && (uint32_t)k < live;
        const int bk = cut_k ? bin_of_count(k) : kFine - 1;
        const bool at_k = bk < kFine - 1;    // (behind it: among the tokens of weight 0, which add nothing)
        const bool at_p = p < 1.f;
        float v = sh.cum_e[kFine - 2], vp = 0.f;
        if (at_k) {
            const uint32_t before = bk ? sh.cum_c[bk - 1] : 0;
            const float eb = bk ? sh.cum_e[bk - 1] : 0.f;
            v = eb + (sh.cum_e[bk] - eb) * (float)((uint32_t)k - before) / (float)(sh.cum_c[bk] - before);
        }
        // the kept sum lies in [v, v_most]: top-p keeps up to a token more than it asks for, min-p some part of a bin
        float v_most = v;
        if (at_p) {
            vp = v * fmaxf(p, 0.f);
            v_most = fminf(v, vp + exp2f(-1.4426950f * s.nats * fmaxf(bin_of_estimate(vp) - 1.f, 0.f)));
            v = vp;
        }
        if (mp > 0.f) {
            const int b = min((int)fminf(-logf(fminf(mp, 1.f)) / s.nats, 1e6f), kFine - 2);
            v = fminf(v, b ? sh.cum_e[b - 1] : 0.f);
            v_most = fminf(v_most, sh.cum_e[min(b + 1, kFine - 2)]);
        }
        Place at[3];   // of the k-th token, of top-p's last, of the one that u picks
        const auto places = [&](int width) {
            at[0] = at_k ? Place{bk, bk} : Place{1, 0};
            at[1] = at_p ? around(vp, width) : Place{1, 0};
            at[2] = Place{around(v * (float)u, width).lo, around(v_most * (float)u, width).hi};
            // (each begins no later than the next, as it should: the sums in front of them are sums of classes)
            if (at_k && at_p) at[1].lo = min(at[1].lo, bk);
            at[2].lo = min(at[2].lo, at_p ? at[1].lo : at_k ? bk : at[2].lo);
            uint32_t n = 0;
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (at[i].lo <= at[i].hi) n += sh.cum_c[at[i].hi] - (at[i].lo ? sh.cum_c[at[i].lo - 1] : 0);
            return n <= kList;
        };
        // the k-th token's bin and all before it, where these fit: no other weight is asked for
        const bool head = at_k && sh.cum_c[bk] <= kList;
        // (the sum, in units of the largest weight, says over how many tokens the errors cancel: 20 times at 400)
        int width = head ? sure : sh.cum_e[kFine - 2] >= 400.f ? narrow : usual;
        if (!places(width)) width = narrow;
        for (; width <= sure; ++width) {
            if (!places(width) && !head) return false;
            if (collect(a, r, k, p, mp, u, least, at, head, at_k, at_p, bk, live)) return true;
        }
        return false;
    }
    __device__ bool collect(const SampleArgs& a, int r, int k, float p, float mp, double u, float least,
                            const Place (&at)[3], bool head, bool at_k, bool at_p, int bk, uint32_t live) {
        // ---- the tokens, and the weights in front of them ----
        u64* list = reinterpret_cast<u64*>(hist);
        if (tid == 0) sh.n_list = 0;
        __syncthreads();
        const auto take = [&](const float(&x)[8], int i, uint32_t in) {
            for (; in; in &= in - 1) {
                const int j = __ffs(in) - 1;
                list[atomicAdd(&sh.n_list, 1u)] = (u64)order_of(pick(x, j)) << 32 | (uint32_t)(i + j);
            }
        };
        u64 all_w = 0, kept_c = 0, kept_w = 0, front[3] = {0, 0, 0};
        if (head) {   // nothing but these matters
            each8([&](const float(&x)[8], int i) {
                uint32_t in = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) in |= (uint32_t)(fine_of(s, x[j]) <= bk) << j;
                take(x, i, in);
            });
        } else {
            // Classes of tokens: in front of u's place, from there to top-p's, from there to the k-th's, behind; a thread sums the
            // weights of each in a column of its own.  A token is taken up to the end of the last place that began.
            const int lo0 = at[2].lo, lo1 = at_p ? at[1].lo : lo0, lo2 = at_k ? bk : lo1;
            const int hi0 = at[2].hi, hi1 = at_p ? max(hi0, at[1].hi) : hi0, hi2 = at_k ? max(hi1, bk) : hi1;
            const uint32_t column = tc::s2u(hist) + kList * 8 + tid * 8;   // (behind the list)
#pragma unroll
            for (int c = 0; c < 4; ++c) sts64(column + c * (kThreads * 8), 0);
            const auto sum_up = [&](auto with_floor) {
                each8([&](const float(&x)[8], int i) {
                    u64 w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = weight_units(s, fmaxf(x[j], s.low));
                    uint32_t in = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int b = fine_of(s, x[j]);
                        const u64 units = b < kFine - 1 ? w[j] : 0;
                        const int c = (b >= lo0) + (b >= lo1) + (b >= lo2);
                        bump(column, c, units);
                        in |= (uint32_t)(b >= lo0 && b <= (b >= lo2 ? hi2 : b >= lo1 ? hi1 : hi0)) << j;
                        if constexpr (decltype(with_floor)::value) {
                            const bool keep = x[j] > -INFINITY && x[j] >= least;
                            kept_c += keep, kept_w += keep ? units : 0;
                        }
                    }
                    take(x, i, in);
                });
            };
            if (mp > 0.f) sum_up(std::true_type{});
            else sum_up(std::false_type{});
            front[2] = lds64(column);
            front[1] = front[2] + lds64(column + kThreads * 8);
            front[0] = front[1] + lds64(column + 2 * kThreads * 8);
            all_w = front[0] + lds64(column + 3 * kThreads * 8);
            block_sum(all_w, front[0]);
            block_sum(front[1], front[2]);
            block_sum(kept_c, kept_w);
        }
        publish(64, all_w), publish(65, front[0]), publish(66, front[1]), publish(67, front[2]), publish(68, kept_c), publish(69, kept_w);
        const u64(*in)[72] = exchange();
        if (rank == 0) {
            all_w = front[0] = front[1] = front[2] = kept_c = kept_w = 0;
            int n_list = (int)sh.n_list;
            for (int q = 0; q < n_ranks; ++q) {
                all_w += in[q][64], front[0] += in[q][65], front[1] += in[q][66], front[2] += in[q][67], kept_c += in[q][68], kept_w += in[q][69];
                if (q == 0) continue;
                const int more = (int)*cluster.map_shared_rank(&sh.n_list, q);
                const u64* from = cluster.map_shared_rank(list, q);
                for (int i = tid; i < more; i += kThreads) list[n_list + i] = from[i];
                n_list += more;
            }
            __syncthreads();
            const bool ok = settle(a, r, k, p, mp, u, least, at, head, live, at_k, n_list, all_w, front, kept_c, kept_w);
            if (tid < n_ranks) *cluster.map_shared_rank(&sh.done, tid) = ok;
        }
        cluster.sync();
        return sh.done;
    }
    // Rank 0: the searches, over the list.  False where an estimate was too far off.
    __device__ bool settle(const SampleArgs& a, int r, int k, float p, float mp, double u, float least,
                           const Place (&at)[3], bool head, uint32_t live, bool at_k, int n_list, u64 all_w, const u64 (&front)[3],
                           u64 kept_c, u64 kept_w) {
        u64 n = k > 0 && (uint32_t)k < live ? k : live, sum = all_w;
        Found f;
        if (at_k) {
            if (!find(true, k, at[0], head, front[0], n_list, f)) return false;
            sum = f.weight;
        }
        if (p < 1.f) {
            const u64 target = reach(p, sum);
            if (!find_weight(target, at[1], head, front[1], n_list, f)) return false;
            if (f.count < n) n = f.count, sum = f.weight;
        }
        if (mp > 1.f) {
            kept_c = 1, kept_w = (u64)s.unit;   // nobody reaches it: the first token alone
        } else if (mp > 0.f && head) {   // (what min-p keeps beyond the k-th does not matter)
            const u64* list = reinterpret_cast<const u64*>(hist);
            kept_c = kept_w = 0;
            for (int i = tid; i < n_list; i += kThreads) {
                const float x = value_of((uint32_t)(list[i] >> 32));
                const u64 units = weight_units(s, fmaxf(x, s.low));
                if (x >= least) kept_c += 1, kept_w += units;
            }
            block_sum(kept_c, kept_w);
        }
        if (mp > 0.f && kept_c < n) n = kept_c, sum = kept_w;
        const u64 target = pass(u, sum);
        if (!find_weight(target, at[2], head, front[2], n_list, f)) return false;
        answer(a, r, f, n, sum);
        return true;
    }
    // (with all tokens at hand, where the target itself says, and a wider place if need be)
    __device__ bool find_weight(u64 target, const Place& place, bool head, u64 front, int n_list, Found& f) {
        if (!head) return find(false, target, place, head, front, n_list, f);
        const float v = (float)((double)target / s.unit);
        return find(false, target, around(v, usual), head, front, n_list, f) || find(false, target, around(v, sure), head, front, n_list, f);
    }
    // search() among the list's tokens of the fine bins of `place`; in front of them stand `front` units of weight, or (head)
    // the list's own tokens of lower bins
    __device__ bool find(bool by_count, u64 target, const Place& place, bool head, u64 front, int n_list, Found& f) {
        const u64* list = reinterpret_cast<const u64*>(hist);
        u64* found = reinterpret_cast<u64*>(hist) + kList;
        __syncthreads();   // the last search's list and counter are done with
        if (tid == 0) sh.n_next = 0;
        __syncthreads();
        u64 before = 0, here = 0;
        constexpr int kMine = kList / kThreads;
        u64 o[kMine], w[kMine];
#pragma unroll
        for (int e = 0; e < kMine; ++e) o[e] = list[e * kThreads + tid];   // (what stands behind the list is not used)
#pragma unroll
        for (int e = 0; e < kMine; ++e) w[e] = weight_units(s, fmaxf(value_of((uint32_t)(o[e] >> 32)), s.low));
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
            const int b = fine_of(s, value_of((uint32_t)(o[e] >> 32)));
            if (e * kThreads + tid >= n_list || b > place.hi || (b < place.lo && !head)) continue;
            const u64 units = b < kFine - 1 ? w[e] : 0;
            if (b < place.lo) {
                before += units;
            } else {
                here += units;
                found[atomicAdd(&sh.n_next, 1u)] = o[e];
            }
        }
        block_sum(before, here);
        if (!head) before = front;
        const u64 count = place.lo ? sh.cum_c[place.lo - 1] : 0;
        const int n = (int)sh.n_next;
        if (n == 0 || (by_count ? target <= count || target > count + n : target <= before || target > before + here)) return false;
        f = select(by_count, target, count, before, found, n);
        return true;
    }
    // f(eight logits, index of the first) for this CTA's segment, out of shared memory where it is kept there (a thread finds its
    // own elements)
    template <typename F>
    __device__ __forceinline__ void each8(F f) {
        for (int i = begin + tid * 8; i < end; i += kThreads * 8) {
            float x[8];
            if constexpr (kResident) {
                constexpr int V = 8 * sizeof(T) / 16;
                uint4 raw[V];
#pragma unroll
                for (int v = 0; v < V; ++v) raw[v] = lds128(kept + (i - begin) * (int)sizeof(T) + v * 16);
                unpack8(raw, i, end, x);
            } else {
                load8(row, i, end, x);
            }
            f(x, i);
        }
    }
    // f(logit, order) for the tokens of a range: of a bin, of a sixteenth of it (sub >= 0), from lo to hi in the order
    struct Range {
        int bin, sub;
        u64 lo, hi;
    };
    template <typename F>
    __device__ __forceinline__ void each_of(const Range& r, F f) {
        const float z0 = r.bin - 0.5f;
        each8([&](const float(&x)[8], int i) {
            uint32_t in = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                in |= (uint32_t)(bin_of(s, x[j]) == r.bin && (r.sub < 0 || part_of(s, x[j], z0, kBins, kBins) == r.sub)) << j;
            for (; in; in &= in - 1) {
                const int j = __ffs(in) - 1;
                const float v = pick(x, j);
                if (!(v > -INFINITY)) continue;
                const u64 o = (u64)order_of(v) << 32 | (uint32_t)(i + j);
                if (o >= r.lo && o <= r.hi) f(v, o);
            }
        });
    }
    static __device__ __forceinline__ float pick(const float (&x)[8], int j) {
        float v = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) v = j == e ? x[e] : v;
        return v;
    }
    // the same over the row itself, four loads under way, leaving the segment in shared memory
    template <typename F>
    __device__ __forceinline__ void first_pass(F f) {
        constexpr int U = 4, V = 8 * sizeof(T) / 16;
        for (int i0 = begin + tid * 8; i0 < end; i0 += U * kThreads * 8) {
            uint4 raw[U][V];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * kThreads * 8;
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (i + v * (8 / V) < end) raw[k][v] = __ldcs(reinterpret_cast<const uint4*>(row + i) + v);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * kThreads * 8;
                if (i >= end) break;
                float x[8];
                unpack8(raw[k], i, end, x);
                if constexpr (kResident) {
#pragma unroll
                    for (int v = 0; v < V; ++v) sts128(kept + (i - begin) * (int)sizeof(T) + v * 16, raw[k][v]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) f(x[j], i + j);
            }
        }
    }
    __device__ __forceinline__ u64 weight_or_0(float x, int bin) const { return bin < kZeroBin ? weight_units(s, x) : 0; }

    __device__ __forceinline__ void block_min_max(u64& a, u64& b) {
        a = warp_min(a), b = warp_max(b);
        __syncthreads();
        if (lane == 0) sh.red_a[warp] = a, sh.red_b[warp] = b;
        __syncthreads();
        a = warp_min(sh.red_a[lane % kWarps]), b = warp_max(sh.red_b[lane % kWarps]);
    }
    __device__ __forceinline__ void block_sum(u64& a, u64& b) {
        a = warp_sum(a), b = warp_sum(b);
        __syncthreads();
        if (lane == 0) sh.red_a[warp] = a, sh.red_b[warp] = b;
        __syncthreads();
        a = warp_sum(lane < kWarps ? sh.red_a[lane] : 0), b = warp_sum(lane < kWarps ? sh.red_b[lane] : 0);
    }
    // the CTA's sums of the bins, to every CTA of the row
    __device__ __forceinline__ void reduce_bins() {
        __syncthreads();
        const u64* h = reinterpret_cast<const u64*>(hist);
        for (int b = warp; b < kBins; b += kWarps) {
            u64 w = 0, c = 0;
#pragma unroll 4
            for (int k = lane; k < kThreads; k += 32) {
                const u64 v = h[b * kThreads + k];
                w += v & ((1ull << kWeightBits) - 1), c += v >> kWeightBits;
            }
            w = warp_sum(w), c = warp_sum(c);
            if (lane < n_ranks) {
                u64(*to)[72] = cluster.map_shared_rank(sh.xch[turn], lane);
                to[rank][b] = w, to[rank][32 + b] = c;
            }
        }
    }
    __device__ __forceinline__ void publish(int slot, u64 v) {
        if (tid < n_ranks) cluster.map_shared_rank(sh.xch[turn], tid)[rank][slot] = v;
    }
    // what every rank has published since the last exchange; stays readable until the exchange after next
    __device__ __forceinline__ const u64 (*exchange())[72] {
        cluster.sync();
        const u64(*in)[72] = sh.xch[turn];
        turn ^= 1;
        return in;
    }

    // the bin in which the running count (or weight) reaches `target`, and what stands in front of it
    __device__ __forceinline__ int bin_reaching(bool by_count, u64 target, u64& base_c, u64& base_w) const {
        base_c = base_w = 0;
        int bin = 0;
        for (; bin < kZeroBin; ++bin) {
            const u64 c = sh.bin_c[bin], w = sh.bin_w[bin];
            if ((by_count ? base_c + c : base_w + w) >= target) break;
            base_c += c, base_w += w;
        }
        return bin;
    }
    // the CTAs' lists of the tokens that `add` puts there, all on rank 0; returns their number there
    template <typename F>
    __device__ __forceinline__ int collect(F each_one) {
        u64* list = reinterpret_cast<u64*>(hist);
        if (tid == 0) sh.n_list = 0;
        __syncthreads();
        each_one([&](u64 o) { list[atomicAdd(&sh.n_list, 1u)] = o; });
        cluster.sync();
        int n = (int)sh.n_list;
        if (rank == 0) {
            for (int k = 1; k < n_ranks; ++k) {
                const int more = (int)*cluster.map_shared_rank(&sh.n_list, k);
                const u64* from = cluster.map_shared_rank(list, k);
                for (int i = tid; i < more; i += kThreads) list[n + i] = from[i];
                n += more;
            }
            __syncthreads();
        }
        return n;
    }
    // The first token, in order, at which the running count (or weight) reaches `target` (1 <= target <= the total).
    __device__ Found search(bool by_count, u64 target) {
        u64 base_c, base_w;
        const int bin = bin_reaching(by_count, target, base_c, base_w);
        if (bin == kZeroBin && by_count) return Found{target, base_w, ~0ull};   // among the tokens of weight 0: nobody asks which
        // the range of the order that holds it, narrowed until its tokens fit a list: by the depth first, then by the order itself
        // (equal logits in the end)
        Range r{bin, -1, 0, ~0ull};
        u64 in_range = sh.bin_c[bin];
        while (in_range > kList) {
            const bool by_depth = r.sub < 0;
            u64 least = 0;
            int shift = 0;
            if (!by_depth) {
                u64 most = 0;
                least = ~0ull;
                each_of(r, [&](float, u64 o) { least = min(least, o), most = max(most, o); });
                block_min_max(least, most);
                publish(64, least), publish(65, most);
                const u64(*in)[72] = exchange();
                least = ~0ull, most = 0;
                for (int k = 0; k < n_ranks; ++k) least = min(least, in[k][64]), most = max(most, in[k][65]);
                shift = max(0, 64 - kBinBits - __clzll((long long)(most - least)));   // half of the parts are used at least
            }
            const uint32_t column = tc::s2u(hist) + tid * 8;
#pragma unroll
            for (int b = 0; b < kBins; ++b) sts64(column + b * (kThreads * 8), 0);
            const float z0 = bin - 0.5f;
            if (by_depth) {
                each8([&](const float(&x)[8], int) {
                    u64 w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = weight_units(s, fmaxf(x[j], s.low));
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (bin_of(s, x[j]) == bin && x[j] > -INFINITY)
                            bump(column, part_of(s, x[j], z0, kBins, kBins), (bin < kZeroBin ? w[j] : 0) + (1ull << kWeightBits));
                });
            } else {
                each_of(r, [&](float x, u64 o) {
                    bump(column, (int)((o - least) >> shift), weight_or_0(x, bin) + (1ull << kWeightBits));
                });
            }
            reduce_bins();
            const u64(*all)[72] = exchange();
            int part = 0;
            for (;; ++part) {
                u64 c = 0, w = 0;
                for (int k = 0; k < n_ranks; ++k) w += all[k][part], c += all[k][32 + part];
                in_range = c;
                if (part == kBins - 1 || (by_count ? base_c + c : base_w + w) >= target) break;
                base_c += c, base_w += w;
            }
            if (by_depth) {
                r.sub = part;
            } else {
                r.lo = least + ((u64)part << shift);
                r.hi = r.lo + ((1ull << shift) - 1);
                if (r.hi < r.lo) r.hi = ~0ull;
            }
        }
        const int n = collect([&](auto put) { each_of(r, [&](float, u64 o) { put(o); }); });
        if (rank == 0) {
            const Found f = select(by_count, target, base_c, base_w, reinterpret_cast<u64*>(hist), n);
            if (tid < n_ranks) *cluster.map_shared_rank(&sh.found, tid) = f;
        }
        cluster.sync();
        return sh.found;
    }

    // the same over a list in shared memory, which is used up; one CTA
    __device__ Found select(bool by_count, u64 target, u64 base_c, u64 base_w, u64* list, int n) {
        constexpr int kMine = kList / kThreads;
        while (n > kFew) {
            u64 least = ~0ull, most = 0, o[kMine];
#pragma unroll
            for (int e = 0; e < kMine; ++e) {
                const int i = e * kThreads + tid;
                o[e] = i < n ? list[i] : ~0ull;
                if (i < n) least = min(least, o[e]), most = max(most, o[e]);
            }
            block_min_max(least, most);
            const int shift = max(0, 56 - __clzll((long long)(most - least)));   // 256 parts, half of them used at least
            if (tid < 256) sh.part_w[tid] = 0, sh.part_c[tid] = 0;
            if (tid == 0) sh.n_next = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kMine; ++e) {
                if (e * kThreads + tid >= n) break;
                const int part = (int)((o[e] - least) >> shift);
                const float x = value_of((uint32_t)(o[e] >> 32));
                atomicAdd(&sh.part_c[part], 1u);
                atomicAdd(&sh.part_w[part], weight_or_0(x, bin_of(s, x)));
            }
            __syncthreads();
            if (warp == 0) {   // the part, by a scan of 8 parts a lane
                u64 w[8], c[8], tw = 0, tc = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = sh.part_w[lane * 8 + k], c[k] = sh.part_c[lane * 8 + k], tw += w[k], tc += c[k];
                u64 pw = tw, pc = tc;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const u64 xw = __shfl_up_sync(0xffffffffu, pw, d), xc = __shfl_up_sync(0xffffffffu, pc, d);
                    if (lane >= d) pw += xw, pc += xc;
                }
                const bool reached = (by_count ? base_c + pc : base_w + pw) >= target;
                const uint32_t m = __ballot_sync(0xffffffffu, reached);
                if (lane == (m ? __ffs(m) - 1 : 31)) {
                    u64 bw = base_w + pw - tw, bc = base_c + pc - tc;
                    int k = 0;
                    for (; k < 7; ++k) {
                        if ((by_count ? bc + c[k] : bw + w[k]) >= target) break;
                        bw += w[k], bc += c[k];
                    }
                    sh.pick[0] = bc, sh.pick[1] = bw, sh.pick[2] = lane * 8 + k;
                }
            }
            __syncthreads();
            base_c = sh.pick[0], base_w = sh.pick[1];
            const int part = (int)sh.pick[2];
#pragma unroll
            for (int e = 0; e < kMine; ++e)
                if (e * kThreads + tid < n && (int)((o[e] - least) >> shift) == part) list[atomicAdd(&sh.n_next, 1u)] = o[e];
            __syncthreads();
            n = (int)sh.n_next;
            __syncthreads();
        }
        // few: every one against every other; four threads a candidate
        if (tid < n) {
            const float x = value_of((uint32_t)(list[tid] >> 32));
            sh.cand_w[tid] = weight_or_0(x, bin_of(s, x));
        }
        __syncthreads();
        const int mine = tid >> 2;
        u64 c = 0, w = 0;
        const u64 me = mine < n ? list[mine] : 0;
        if (mine < n)
            for (int i = tid & 3; i < n; i += 4)
                if (list[i] <= me) c += 1, w += sh.cand_w[i];
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            c += __shfl_xor_sync(0xffffffffu, c, o);
            w += __shfl_xor_sync(0xffffffffu, w, o);
        }
        if (mine < n && (tid & 3) == 0) {
            const u64 own = sh.cand_w[mine];
            const bool here = by_count ? base_c + c == target : base_w + w >= target && base_w + w - own < target;
            if (here) sh.pick[0] = base_c + c, sh.pick[1] = base_w + w, sh.pick[2] = me;
        }
        __syncthreads();
        const Found f{sh.pick[0], sh.pick[1], sh.pick[2]};
        return f;
    }
};

template <typename T, bool kResident>
__global__ void __launch_bounds__(kThreads, kResident ? 1 : 2) sample_kernel(const SampleArgs a, int segment) {
    extern __shared__ __align__(16) unsigned char hist[];   // the bins (or lists), then the segment
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    tc::cluster_arrive_relaxed();   // "this CTA has started"; run() waits for the others' behind the first pass over the row
    for (int i = threadIdx.x; i < 64 * 16; i += kThreads) sh.tab.v[i >> 4][i & 15] = exp2((double)(i >> 4) / 64.0);
    tc::pdl_wait();
    tc::pdl_launch_dependents();
    __syncthreads();
    const int n_ranks = cluster.num_blocks(), r = blockIdx.x / n_ranks;
    const int begin = min((int)cluster.block_rank() * segment, a.vocab), end = min(begin + segment, a.vocab);
    RowSampler<T, kResident> row(sh, hist, tc::s2u(hist + HIST_BYTES), static_cast<const T*>(a.logits) + r * a.row_stride, begin, end);
    row.run(a, r);
    cluster.sync();   // no CTA leaves while another may still write into its shared memory
}

template <typename T, bool kResident>
cudaError_t launch_as(const SampleArgs& a, int c, int segment, cudaStream_t stream) {
    const int bytes = (int)HIST_BYTES + (kResident ? segment * (int)sizeof(T) : 0);
    static PerDeviceOnce once;
    if (const cudaError_t e = ensure_dynamic_smem(once, sample_kernel<T, kResident>, kResident ? kMaxDynamic : (int)HIST_BYTES); e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.n_rows * c, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = c;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T, kResident>, a, segment);
}

// CTAs of a row, and whether a segment is kept in shared memory (one CTA an SM) or read again from L2 (two).  Kept, a CTA takes
// 14 us and 0.8 us for each 1000 tokens, and the CTAs that do not fit at once make whole further rounds while these are few.  Read
// again, 14 and 1.05 alone on an SM, 22 and 1.5 in pairs; in a single round the slowest rows count, 18 and 2.1.  From 16384
// columns on a row has two CTAs at least: what one does by itself is the longer part of a slow row.
// us, kept with 2 / 4 / 8 CTAs, read again with 2 / 4 / 8: 32 rows of 126464 in fp32 69 40 53, 69 47 46; 256 rows of 152064 in bf16
// (not kept with 2) - 300 460, 281 266 -; 128 of 126464 in bf16 120 115 192, 148 110 143; 128 of 32000 49 74 150, 53 58 109 (one
// CTA 69, 78); 64 of 126464 in fp32 90 81 130, 90 76 97; 16 of 152064 in bf16 102 73 62, 102 80 71.
template <typename T>
cudaError_t launch(const SampleArgs& a, cudaStream_t stream) {
    const auto segment = [&](int c) { return ((a.vocab + c - 1) / c + 7) & ~7; };
    const double sms = sm_count();
    int best_c = kMaxCluster;
    bool kept = false;
    double best = 1e30;
    for (int c = a.vocab < 16384 ? 1 : 2; c <= kMaxCluster; c *= 2) {
        const int seg = segment(c);
        if (seg > kSegment || (c > 1 && seg < 1024)) continue;
        const double ctas = (double)a.n_rows * c;
        if ((int)HIST_BYTES + (long long)seg * (int)sizeof(T) <= kMaxDynamic) {
            const double rounds = ctas / sms, us = (14. + 8e-4 * seg) * (rounds <= 3. ? ceil(rounds) : rounds);
            if (us < best) best = us, best_c = c, kept = true;
        }
        const double once = 18. + 2.1e-3 * seg, more = ctas / (2. * sms) * (22. + 1.5e-3 * seg);
        const double us = ctas <= sms ? 14. + 1.05e-3 * seg : once > more ? once : more;
        if (us < best) best = us, best_c = c, kept = false;
    }
    return kept ? launch_as<T, true>(a, best_c, segment(best_c), stream) : launch_as<T, false>(a, best_c, segment(best_c), stream);
}

}  // namespace

size_t sample_workspace_bytes(int, int) { return 16; }   // everything stays in shared memory

cudaError_t launch_sample(const SampleArgs& a, cudaStream_t stream) {
    return a.dtype == EC_BF16 ? launch<__nv_bfloat16>(a, stream) : launch<float>(a, stream);
}

}  // namespace ec
