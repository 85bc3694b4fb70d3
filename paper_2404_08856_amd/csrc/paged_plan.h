// How the workgroups of the attention kernels over pages share the work, found by each of them from the lengths in device memory.
//
// The query heads of a key head are taken together: row i and head j of the group of `group` make packed row i * group + j, and QT packed rows of a
// (sequence, key head) make a tile.  A tile's cost is about the number of keys that its last row sees, so that the sum over a sequence's tiles has a closed
// form; all tiles in a row (sequences, key heads, tiles) are cut into W runs of equal cost.  A workgroup takes the tiles or parts of tiles of its run.  A tile
// that several workgroups share is joined by the last of them to arrive: each leaves its unnormalised sums and its maximum in a slot of the
// workspace, then puts the call's number on the slot's flag, then looks whether all flags of the tile carry it.  Nobody waits.
#pragma once
#include "paged.h"

namespace spd {

typedef unsigned long long u64;

// lane l's value, in scalar registers
__device__ __forceinline__ u64 lane_value(u64 x, int l) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, l);
}

struct PagedPlan {
    u64 number;              // of the call: what a flag of this call carries
    u64 least;               // cost of a workgroup at least
    int group;               // query heads of a key head
    int above, upto;         // takes the sequences with so many packed rows: above < rows <= upto
    u64 *flags;              // [2 * workgroups]
    float *slots;            // [2 * workgroups][QT * (dim + 2)]
};

// A sequence as one kernel sees it
template <int QT>
struct PagedSeq {
    static constexpr int kStart = 64;      // cost of a tile besides its keys
    int first, n, len, tiles, rising;
    unsigned rows;                         // rows a tile covers, rounded up
    u64 most;
    __device__ __forceinline__ void init(const PagedAttentionArgs &a, const PagedPlan &pl, int s) {
        int last;
        paged_rows(a.b, s, first, last);
        n = last - first;
        len = paged_len(a.b, s);
        const int packed = n * pl.group;
        tiles = packed > pl.above && packed <= pl.upto ? (packed + QT - 1) / QT : 0;
        rows = (QT + pl.group - 1) / pl.group;
        most = a.window ? (u64)a.window + rows : ~0ull >> 8;
        rising = most > (u64)len ? (int)min((u64)tiles, (most - len) / rows) : 0;
    }
    __device__ __forceinline__ u64 cost(int t) const { return min(len + (u64)(t + 1) * rows, most) + kStart; }
    __device__ __forceinline__ u64 before(int t) const {       // sum of the costs of tiles 0 .. t - 1
        const u64 c = min(t, rising);
        return c * (len + kStart) + rows * (c * (c + 1) / 2) + (u64)(t - c) * (most + kStart);
    }
    __device__ __forceinline__ int tile_at(u64 x) const {      // the tile that the cost x < before(tiles) falls into
        int lo = 0, hi = tiles;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (before(mid) <= x) lo = mid; else hi = mid;
        }
        return lo;
    }
};

// The runs: workgroup w takes [start(w), start(w + 1)) of the whole cost
struct PagedRuns {
    u64 each, more;
    int n;                                 // workgroups
    __device__ __forceinline__ void init(u64 total, u64 least, int groups) {
        n = (int)max(1ull, min((u64)groups, total / least));
        each = total / n;
        more = total - each * n;           // the first `more` workgroups take one more
    }
    __device__ __forceinline__ u64 start(int w) const { return each * w + min((u64)w, more); }
    __device__ __forceinline__ int of(u64 x) const {
        const u64 line = more * (each + 1);
        return (int)(x < line ? x / (each + 1) : more + (x - line) / each);
    }
};

// Called by whole waves.  total: cost of all sequences; at(x): the sequence that cost x falls into, and the cost before it.
template <int QT>
struct PagedMap {
    const PagedAttentionArgs &a;
    const PagedPlan &pl;
    __device__ __forceinline__ PagedMap(const PagedAttentionArgs &a_, const PagedPlan &p_) : a(a_), pl(p_) {}
    __device__ __forceinline__ u64 cost_of(int s) const {
        if (s >= a.b.n_seqs) return 0;
        PagedSeq<QT> q;
        q.init(a, pl, s);
        return q.tiles ? q.before(q.tiles) * a.c.n_kv : 0;
    }
    __device__ __forceinline__ static u64 scan(u64 x, int lane) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const u64 y = __shfl_up(x, d);
            if (lane >= d) x += y;
        }
        return x;
    }
    __device__ __forceinline__ u64 total(u64 &mine) const {      // mine: this lane's prefix over the first 64 sequences, itself included
        const int lane = threadIdx.x & 63;
        mine = scan(cost_of(lane), lane);
        u64 sum = lane_value(mine, 63);
        for (int s = 64; s < a.b.n_seqs; s += 64) sum += lane_value(scan(cost_of(s + lane), lane), 63);
        return sum;
    }
    __device__ __forceinline__ void at(u64 x, u64 mine, int &s, u64 &before) const {
        const int lane = threadIdx.x & 63;
        u64 base = 0;
        for (int s0 = 0;; s0 += 64) {
            const u64 upto = (s0 ? scan(cost_of(s0 + lane), lane) : mine) + base;
            const u64 hit = __ballot(upto > x);
            if (hit || s0 + 64 >= a.b.n_seqs) {
                const int l = hit ? __builtin_ctzll(hit) : 63;   // (x is below the total: there is a hit)
                s = s0 + l;
                before = l ? lane_value(upto, l - 1) : base;
                return;
            }
            base = lane_value(upto, 63);
        }
    }
};

}  // namespace spd
