// How the workgroups of the attention kernels over pages share the work, found by each of them from the lengths in device memory.
//
// The query heads of a key head are taken together: row i and head j of the group of `group` make packed row i * group + j, and QT packed rows of a
// (sequence, key head) make a tile.  A tile's cost is about the number of keys that its last row sees, so that the sum over a sequence's tiles has a closed
// form; all tiles in a row (sequences, key heads, tiles) are cut into W runs of equal cost.  A workgroup takes the tiles or parts of tiles of its run.  A tile
// that several workgroups share is joined by the last of them to arrive: each leaves its unnormalised sums and its maximum in a slot of the
// workspace, then puts the call's number on the slot's flag, then looks whether all flags of the tile carry it.  Nobody waits.  (Two may find them all there: both write
// the same.)  The flags are cleared by who has joined, so that a replay of the same call begins with none.
//
// A shared tile costs about 5 us with few rows and 10 with many, beside what it divides: so tiles are shared only where that is expected to pay (PagedRuns).  One token of
// 640 keys in 32 heads 25.6 us shared over 120 workgroups, 19.1 over 36, 12.5 by a workgroup a head; 64 uneven sequences 190 us shared and 230 by a workgroup a tile.
#pragma once
#include "paged.h"

namespace spd {

typedef unsigned long long u64;

struct PagedPlan {
    u64 number;              // of the call: what a flag of this call carries
    unsigned least;          // cost of a workgroup at least
    unsigned join;           // what sharing a tile costs
    int shift;               // a cost counts 2^shift keys, so that the whole fits 31 bits
    int group;               // query heads of a key head
    int above, upto;         // takes the sequences with so many packed rows: above < rows <= upto
    u64 *flags;              // [2 * workgroups]
    float *slots;            // [2 * workgroups][QT * (dim + 3)]
};

// A sequence as one kernel sees it
template <int QT>
struct PagedSeq {
    int first, n, len, tiles, rising;
    unsigned base, rows, most, whole;      // cost of tile t: min(base + (t + 1) rows, most) + 1; of all tiles: whole
    // flat: every tile costs 1
    __device__ __forceinline__ void init(const PagedAttentionArgs &a, const PagedPlan &pl, int s, bool flat) {
        int last;
        paged_rows(a.b, s, first, last);
        n = last - first;
        len = paged_len(a.b, s);
        const int packed = n * pl.group;
        tiles = packed > pl.above && packed <= pl.upto ? (packed + QT - 1) / QT : 0;
        const unsigned span = (QT + pl.group - 1) / pl.group;               // rows a tile covers, rounded up
        base = (unsigned)(len + kStart) >> pl.shift;
        rows = span >> pl.shift;
        most = a.window ? ((unsigned)a.window + span + kStart) >> pl.shift : 0x7fffffffu;
        if (flat) base = rows = 0;
        rising = most < base ? 0 : (rows && a.window ? (int)min((unsigned)tiles, (most - base) / rows) : tiles);
        whole = before(tiles);
    }
    // What a tile costs besides its keys (its start and its results, in keys).  With 0 uneven batches take more (64 x 1 row 205 us, 191; 33 x 1 to 20 rows 190, 178), with
    // twice as much 17 short prompts 69 (53).
    static constexpr int kStart = QT >= 64 ? 160 : 256;
    // the tile at cost x < whole * heads of the sequence: head, tile, and the cost before it
    __device__ __forceinline__ void at(unsigned x, int heads, bool flat, int &h, int &t, unsigned &first_cost) const {
        if (flat) {
            t = tiles - 1 - (int)(x / (unsigned)heads);
            h = (int)(x % (unsigned)heads);
            first_cost = x;
        } else {
            h = (int)(x / whole);
            t = tile_at(x - h * whole);
            first_cost = h * whole + before(t);
        }
    }
    __device__ __forceinline__ unsigned cost(int t) const { return min(base + (unsigned)(t + 1) * rows, most) + 1; }
    __device__ __forceinline__ unsigned before(int t) const {       // sum of the costs of tiles 0 .. t - 1
        const unsigned c = min(t, rising);
        return c * (base + 1) + rows * (c * (c + 1) / 2) + (unsigned)(t - (int)c) * (most + 1);
    }
    __device__ __forceinline__ int tile_at(unsigned x) const {      // the tile that the cost x < whole falls into
        int lo = 0, hi = tiles;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (before(mid) <= x) lo = mid; else hi = mid;
        }
        return lo;
    }
};

// Of `units` units of a tile those before its cost x (the same for whoever asks; all of them at x = cost)
__device__ __forceinline__ int units_before(int units, unsigned x, unsigned cost) {
    return x >= cost ? units : min(units, (int)((float)x * ((float)units / (float)cost)));
}

// The runs: workgroup w < n takes [start(w), start(w + 1)) of the whole cost.  Where the tiles taken one by one, a sequence's longest first, are expected to be
// done no later than even runs and what sharing tiles costs, each workgroup takes one tile (flat): the expectation is a full round for tiles of about
// the same cost, and, where every sequence's costs fall to half or less, that the short ones fill the gaps.  Called by whole waves.
// side: workgroups that run side by side; grid: all.
template <int QT>
struct PagedRuns {
    const PagedAttentionArgs &a;
    const PagedPlan &pl;
    unsigned each, more, mine = 0;         // mine: this lane's sum of costs over the first 64 sequences, itself included
    int n;                                 // workgroups
    bool flat;

    struct Add { __device__ __forceinline__ unsigned operator()(unsigned x, unsigned y) const { return x + y; } };
    struct Max { __device__ __forceinline__ unsigned operator()(unsigned x, unsigned y) const { return max(x, y); } };
    template <class Op>
    __device__ __forceinline__ static unsigned over_lanes(unsigned x, Op op) {
        x = xor_step<32>(x, op); x = xor_step<16>(x, op); x = xor_step<8>(x, op); x = xor_step<4>(x, op); x = xor_step<2>(x, op);
        return value(xor_step<1>(x, op), 0);
    }
    __device__ __forceinline__ static unsigned value(unsigned x, int l) { return (unsigned)__builtin_amdgcn_readlane((int)x, l); }
    __device__ __forceinline__ static unsigned scan(unsigned x) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const unsigned y = __shfl_up(x, d);
            if (lane >= d) x += y;
        }
        return x;
    }
    __device__ __forceinline__ unsigned cost_of(int s) const {
        if (s >= a.b.n_seqs) return 0;
        PagedSeq<QT> q;
        q.init(a, pl, s, flat);
        return q.whole * a.c.n_kv;
    }
    struct Min { __device__ __forceinline__ unsigned operator()(unsigned x, unsigned y) const { return min(x, y); } };
    __device__ __forceinline__ PagedRuns(const PagedAttentionArgs &a_, const PagedPlan &p_, unsigned side, unsigned grid) : a(a_), pl(p_), flat(false) {
        const int lane = threadIdx.x & 63;
        unsigned total = 0, tiles = 0, largest = 0, least = 0xffffffffu;
        bool falls = true;                 // in every sequence
        if (a.b.n_seqs == 1) {
            PagedSeq<QT> q;
            q.init(a, pl, 0, false);
            tiles = q.tiles;
            total = q.whole * a.c.n_kv;
            largest = q.tiles ? q.cost(q.tiles - 1) : 0;
            least = q.cost(0);
            falls = 2 * least <= largest;
        } else {
            for (int s0 = 0; s0 < a.b.n_seqs; s0 += 64) {
                PagedSeq<QT> q;
                q.tiles = 0; q.whole = 0;
                if (s0 + lane < a.b.n_seqs) q.init(a, pl, s0 + lane, false);
                if (s0 == 0) mine = q.whole * a.c.n_kv;
                total += over_lanes(q.whole * a.c.n_kv, Add());
                tiles += over_lanes(q.tiles, Add());
                largest = max(largest, over_lanes(q.tiles ? q.cost(q.tiles - 1) : 0u, Max()));
                least = min(least, over_lanes(q.tiles ? q.cost(0) : 0xffffffffu, Min()));
                falls = falls && __all(q.tiles == 0 || 2 * q.cost(0) <= q.cost(q.tiles - 1));
            }
        }
        const unsigned items = tiles * a.c.n_kv;
        const unsigned even = total / side, rounds = (items + side - 1) / side;
        const unsigned expected = rounds > 1 && falls ? max(largest, even + least) : rounds * largest;
        flat = items <= grid && expected <= even + pl.join;
        if (flat) total = items;
        n = total == 0 ? 0 : (flat ? (int)items : (int)max(1u, min(side, total / pl.least)));
        each = n ? total / (unsigned)n : 1;
        more = n ? total - each * n : 0;
        if (a.b.n_seqs > 1 && n) mine = scan(flat ? cost_of(lane) : mine);
    }
    __device__ __forceinline__ unsigned start(int w) const { return each * w + min((unsigned)w, more); }
    __device__ __forceinline__ int of(unsigned x) const {          // the workgroup whose run has x
        const unsigned line = more * (each + 1);
        return (int)(x < line ? x / (each + 1) : more + (x - line) / each);
    }
    // the sequence that cost x falls into, and the cost before it
    __device__ __forceinline__ void at(unsigned x, int &s, unsigned &before) const {
        s = 0;
        before = 0;
        if (a.b.n_seqs == 1) return;
        const int lane = threadIdx.x & 63;
        unsigned base = 0;
        for (int s0 = 0;; s0 += 64) {
            const unsigned upto = (s0 ? scan(cost_of(s0 + lane)) : mine) + base;
            const u64 hit = __ballot(upto > x);
            if (hit || s0 + 64 >= a.b.n_seqs) {
                const int l = hit ? __builtin_ctzll(hit) : 63;     // (x is below the whole: there is a hit)
                s = s0 + l;
                before = l ? value(upto, l - 1) : base;
                return;
            }
            base = value(upto, 63);
        }
    }
};

}  // namespace spd
