// How the attention kernels over pages cut their work, on the device: nothing about lengths is known on the host.
//
// The query rows of a kv head (rows of the sequence x its H_q / H_kv query heads, "packed", the query head fastest) are
// taken in tiles of `tm`; a unit is one tile of one kv head of one sequence and takes as many steps as there are key
// tiles of `tk` keys below the highest limit of its rows (one step where it sees nothing: the zeros are written there).
// All units' costs (steps, and a constant for the start and end of a unit), in the order (sequence, kv head, row tile), form
// one line that is cut into equal pieces, one for each CTA.  A unit that a cut divides leaves un-normalised partial rows in the workspace, which a second launch joins:
// every CTA has at most one unit that began before it (slot 0) and one that goes on behind it (slot 1).
#pragma once

#include "ec_common.cuh"

namespace ec {
namespace paged {

struct Plan {
    const int32_t* row_offsets;
    const int32_t* kv_lens;
    int batch, n_rows, max_rows, max_kv;
    int group, n_kv_heads, mask_block;
    int tm, tk;
    int start;       // what a unit costs beside its steps, in steps: its place on the line is that much longer
    int whole;       // 1: cuts stand between units only, nothing is joined
    int min_steps;   // a CTA is given at least this much of the line, fewer CTAs work where there is not enough
    int32_t* dev_status;
};

struct Seq {
    int row0, n, kv;
};
// a / b for a >= 0, b > 0: a division of 64 bits takes several times as long as one of 32
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return (unsigned long long)(a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
__device__ __forceinline__ Seq seq_of(const Plan& p, int b) {
    const int r0 = min(max(p.row_offsets[b], 0), p.n_rows), r1 = min(max(p.row_offsets[b + 1], r0), p.n_rows);
    return Seq{r0, min(r1 - r0, p.max_rows), min(max(p.kv_lens[b], 0), p.max_kv)};
}
__device__ __forceinline__ bool seq_is_cut(const Plan& p, int b, const Seq& s) {
    return p.row_offsets[b + 1] - p.row_offsets[b] != s.n || p.kv_lens[b] != s.kv;
}
// keys that row i of the sequence sees
__device__ __forceinline__ int limit_of(const Plan& p, const Seq& s, int i) {
    if (p.mask_block == 0) return s.kv;
    const int pos = s.kv - s.n + i;
    if (pos < 0) return 0;
    if (p.mask_block == 1) return pos + 1;
    const long long lim = ((long long)(pos / p.mask_block) + 1) * p.mask_block;
    return lim < s.kv ? (int)lim : s.kv;
}
__device__ __forceinline__ int tiles_of(const Plan& p, const Seq& s) {
    return (int)quotient((long long)s.n * p.group + p.tm - 1, p.tm);
}
// steps of row tile `rt` (limits ascend with the row, so the last row of the tile has the highest)
__device__ __forceinline__ int steps_of(const Plan& p, const Seq& s, int rt) {
    const long long last = min((long long)(rt + 1) * p.tm, (long long)s.n * p.group) - 1;
    const int lim = limit_of(p, s, (int)quotient(last, p.group));
    return max(1, (lim + p.tk - 1) / p.tk);
}

struct Unit {
    int b, head, tile;
    Seq s;
    long long w0;   // where it begins on the line
    int steps;
};

// begin[b] = where sequence b begins on the line, begin[batch] = its end; called by the whole CTA
__device__ __forceinline__ void lay_out(const Plan& p, long long* begin) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (p.mask_block == 0) {
        for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
            const Seq s = seq_of(p, b);
            begin[b + 1] = s.n > 0 ? (long long)tiles_of(p, s) * (steps_of(p, s, 0) + p.start) * p.n_kv_heads : 0;
        }
    } else {
        for (int b = warp; b < p.batch; b += warps) {
            const Seq s = seq_of(p, b);
            const int tiles = tiles_of(p, s);
            long long sum = 0;
            for (int t = lane; t < tiles; t += 32) sum += steps_of(p, s, t) + p.start;
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) begin[b + 1] = sum * p.n_kv_heads;
        }
    }
    if (p.dev_status && blockIdx.x == 0)
        for (int b = threadIdx.x; b < p.batch; b += blockDim.x)
            if (seq_is_cut(p, b, seq_of(p, b))) atomicExch(p.dev_status, (int)EC_ERR_SHAPE);
    __syncthreads();
    if (warp == 0) {
        long long carry = 0;
        for (int b0 = 0; b0 < p.batch; b0 += 32) {
            long long v = b0 + lane < p.batch ? begin[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (b0 + lane < p.batch) begin[b0 + lane + 1] = carry + v;
            carry += __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) begin[0] = 0;
    }
    __syncthreads();
}

// the unit at place `w` (0 <= w < all) of the line; called by whole warps, every lane gets it
// (one copy of the code: run once or twice, it takes as long as its fetching)
static __device__ __noinline__ Unit unit_at(const Plan& p, const long long* begin, long long w) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = p.batch - 1;   // the last sequence that begins at or before w (empty ones end where they begin)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (begin[mid] <= w) lo = mid; else hi = mid - 1;
    }
    Unit u;
    u.b = lo;
    u.s = seq_of(p, lo);
    const long long per_head = quotient(begin[lo + 1] - begin[lo], p.n_kv_heads), at = w - begin[lo];
    u.head = (int)quotient(at, per_head);
    const long long in_head = at - u.head * per_head, head0 = begin[lo] + u.head * per_head;
    if (p.mask_block == 0) {
        u.steps = steps_of(p, u.s, 0);
        u.tile = (int)quotient(in_head, u.steps + p.start);
        u.w0 = head0 + (long long)u.tile * (u.steps + p.start);
        return u;
    }
    const int tiles = tiles_of(p, u.s);
    long long done = 0;
    u.tile = 0, u.steps = 1, u.w0 = head0;
    for (int t0 = 0; t0 < tiles; t0 += 32) {
        const int mine = t0 + lane < tiles ? steps_of(p, u.s, t0 + lane) + p.start : 0;
        int run = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += x;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, done + run > in_head);
        if (past) {
            const int first = __ffs(past) - 1;
            u.tile = t0 + first;
            u.steps = __shfl_sync(0xffffffffu, mine, first) - p.start;
            u.w0 = head0 + done + __shfl_sync(0xffffffffu, run, first) - u.steps - p.start;
            break;
        }
        done += __shfl_sync(0xffffffffu, run, 31);
    }
    return u;
}

// the unit behind u on the line (there is one: the caller has steps left)
__device__ __forceinline__ void step_unit(const Plan& p, Unit& u) {
    u.w0 += u.steps + p.start;
    if (++u.tile == tiles_of(p, u.s)) {
        u.tile = 0;
        if (++u.head == p.n_kv_heads) {
            u.head = 0;
            do {
                ++u.b;
                u.s = u.b < p.batch ? seq_of(p, u.b) : Seq{0, 1, 0};
            } while (u.s.n == 0);
        }
    }
    u.steps = steps_of(p, u.s, u.tile);
}

// the first step of a unit that a stretch of the line from `w` on takes (to: the step before which one that ends at w stops)
__device__ __forceinline__ int step_at(const Plan& p, const Unit& u, long long w) {
    const long long in = w - u.w0 - p.start;
    return in <= 0 ? 0 : in >= u.steps ? u.steps : (int)in;
}
// CTAs that get work
__device__ __forceinline__ int workers(const Plan& p, long long all, int ctas) {
    const long long n = quotient(all + p.min_steps - 1, p.min_steps);
    return (int)min((long long)ctas, max(n, 1ll));
}
// Start of a CTA's stretch, and the unit that it falls into
struct Cut {
    long long w;    // on the line, its end where there is nothing left
    long long w0;   // where the unit begins (w0 < w: the cut divides it), -1 where there is nothing left
    int steps, head, tile, row0, n, pad;
};
__device__ __forceinline__ Cut cut_of_end(long long all) { return Cut{all, -1, 0, 0, 0, 0, 0, 0}; }
// The cut before CTA c of `n`.  One that would leave a quarter of its unit or less on one side is moved to that end of the unit
// where the steps allow it (the partial rows of a unit cost about as much as a step).
// (start_unit: the unit that a stretch from this cut on begins with)
__device__ __forceinline__ Cut cut_of(const Plan& p, const long long* begin, long long all, int n, int c, Unit* start_unit) {
    if (c >= n || all == 0) return cut_of_end(all);
    const long long per = quotient(all, n);
    long long w = c <= 0 ? 0 : per * c + quotient((all - per * n) * c, n);
    const Unit u = unit_at(p, begin, w);
    const int in = (int)(w - u.w0);
    if (in > 0) {
        const int slack = u.steps / 4 < p.min_steps / 2 ? u.steps / 4 : p.min_steps / 2, cost = u.steps + p.start;
        if (p.whole || in <= p.start + slack) w = u.w0;
        else if (cost - in <= slack) w = u.w0 + cost;
    }
    if (start_unit && (threadIdx.x & 31) == 0) {
        Unit v = u;
        if (w >= u.w0 + u.steps + p.start && w < all) step_unit(p, v);
        *start_unit = v;
    }
    const bool inside = w < u.w0 + u.steps + p.start;   // (at the end of a unit nothing is divided)
    return Cut{w, inside ? u.w0 : w, u.steps, u.head, u.tile, u.s.row0, u.s.n, 0};
}

}  // namespace paged
}  // namespace ec
