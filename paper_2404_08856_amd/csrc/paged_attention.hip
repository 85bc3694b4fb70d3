// Attention of the new rows of sequences over their pages, on the matrix cores.
//
//   scores   S[key, row] = sum_d K[key, d] q[row, d]      v_mfma_f32_16x16x32_bf16, A = 16 keys x 32 dims, B = q
//   softmax  running maximum and sum per row, in base 2
//   output   O[d, row] = sum_key V[key, d] p[row, key]    A = 16 dims x 32 keys, B = p
//
// float32 rows: q and p as three bf16 terms each, exact to float32's roundings.  bfloat16 rows: p, unnormalised, as two terms where tiles have up to 32 rows (each
// weight within 2^-16 of itself; that kernel waits for memory, and the second product costs it nothing: 8 x 8 rows of 32 heads on 8, 4000 keys, 43 us with either), and as one
// (within 2^-8) where they have more: there the second takes registers or the matrix core's time (16 x 16 rows, 4000 e4m3 keys, 76 us and 100; a prompt of 4096 rows 173 and
// 213).  The roundings of a row's weights need not be independent: one key may outweigh the others, or all scores be equal.  So results of one term are divided by the sum of
// the rounded weights, and are off by at most 2^-8 of the weighted mean of |v - result|, less than their own rounding unless the values scatter widely; lse has the sum from before
// the rounding.  Sums, maxima and statistics are float32 throughout.  e4m3 keys and values are bf16 values, their scales one factor
// of a head's scores and of its output.  The rows of the score tiles are keys in such an order that a lane ends with the weights of a whole granule
// of keys, the 16 bytes of V that it reads for the second product: no data moves between lanes, and every load is 16 bytes of one granule.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "paged_plan.h"

namespace spd {

__device__ __forceinline__ f32x4_t mfma(const uint4 &a, const uint4 &b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) float f32x2_t;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
// c + the two bf16 of x
__device__ __forceinline__ float add_two(uint32_t x, float c) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), c, false);
}
// four e4m3 as four bf16, exactly
__device__ __forceinline__ uint2 wider(uint32_t x) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true);
    return uint2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
// half `e` of a granule (8 elements) as an operand
template <class C>
__device__ __forceinline__ uint4 operand(const uint4 &x, int e) {
    if constexpr (sizeof(C) == 2) return x;
    const uint2 a = wider(e ? x.z : x.x), b = wider(e ? x.w : x.y);
    return uint4{a.x, a.y, b.x, b.y};
}
__device__ __forceinline__ void agent_store(float *p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float agent_load(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A slot of the workspace: QT rows' sums, then their maxima, sums of weights, and of the weights as they are multiplied
constexpr int slot_floats(int QT, int dim) { return QT * (dim + 3); }
constexpr int kFewGroups = 256, kGroups = 512;        // workgroups that share tiles, at most: one or two a CU
constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;

// 8 neighbouring elements of a query as bf16 terms
template <int NT>
__device__ __forceinline__ void load_query(const PagedAttentionArgs &a, size_t at, bool wide, uint4 (&t)[NT]) {
    if constexpr (NT == 1) {
        const uint16_t *p = (const uint16_t *)a.q.p + at;
        if (wide) t[0] = *reinterpret_cast<const uint4 *>(p);
        else t[0] = uint4{p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16, p[6] | (uint32_t)p[7] << 16};
    } else {
        const float *p = (const float *)a.q.p + at;
        float x[8];
        if (wide) {
            *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(p);
            *reinterpret_cast<float4 *>(x + 4) = *reinterpret_cast<const float4 *>(p + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
        uint32_t w[4][kTerms];
#pragma unroll
        for (int i = 0; i < 4; ++i) split3_pair(x[2 * i], x[2 * i + 1], w[i]);
#pragma unroll
        for (int i = 0; i < kTerms; ++i) t[i] = uint4{w[0][i], w[1][i], w[2][i], w[3][i]};
    }
}

// four neighbouring elements of an output row
template <int NT>
__device__ __forceinline__ void store_output(const PagedAttentionArgs &a, size_t at, bool wide, const float (&y)[4]) {
    if constexpr (NT == 1) {
        uint16_t *p = (uint16_t *)a.out.p + at;
        if (wide) *reinterpret_cast<uint2 *>(p) = uint2{two_bf16(y[0], y[1]), two_bf16(y[2], y[3])};
        else for (int i = 0; i < 4; ++i) p[i] = f32_to_bf16_bits(y[i]);
    } else {
        float *p = (float *)a.out.p + at;
        if (wide) *reinterpret_cast<float4 *>(p) = float4{y[0], y[1], y[2], y[3]};
        else for (int i = 0; i < 4; ++i) p[i] = y[i];
    }
}

// What rows of a tile see: keys lo .. hi - 1, and of the new rows those whose bit is set
struct Sees {
    int lo, hi;
    u64 bits;
    __device__ __forceinline__ void init(const PagedAttentionArgs &a, const int first, const int len, const int i) {
        const int p = len + i;
        lo = a.window ? max(0, p - a.window + 1) : 0;
        hi = a.seen ? len : min(p + 1, a.b.capacity);
        bits = a.seen ? a.seen[first + i] : 0;
    }
    // bits of the keys key .. key + n - 1 (n <= 16) that the row sees, of those below `end`
    __device__ __forceinline__ uint32_t keys(int key, int n, int len, int end) const {
        uint32_t m = ((1u << min(max(hi - key, 0), n)) - 1) & ~((1u << min(max(lo - key, 0), n)) - 1);
        if (bits) {
            const int shift = key - len;
            const u64 b = shift >= 0 ? (shift < 64 ? bits >> shift : 0) : (shift > -n ? bits << -shift : 0);
            m |= (uint32_t)b & ((1u << min(max(end - key, 0), n)) - 1);
        }
        return m;
    }
};

// ---- few rows: the waves of a workgroup share a tile's keys ----------------------------------------
// A wave takes units of four granules of keys (32 in bf16, 64 in e4m3), one in NW of the workgroup's run.  The registers of K and V are filled again for the
// wave's next unit as soon as the product has read them, straight from memory: 16 KiB a wave and 128 KiB a CU are under way at any time.
//
// Bound by memory: 64 sequences of 100 to 8000 keys, 32 heads on 8 of 128, one row each, bf16, 190 us, 5.6 TB/s; trees of 9 to 16 rows of 8 sequences of 1500
// to 2047 keys, 32 heads, float32, 50 us, 4.7 TB/s; 4 sequences of 60000 to 131000 keys in e4m3 163 us, 4.8 TB/s.  A single row of 640 keys is a chain of
// latencies, 11.8 us: a start of 1.2, entries of the page table and first keys 3, three rounds of units 4, joining the waves 2.
// Eight waves of at most 256 registers: with the queries in registers instead of LDS, four waves a workgroup and two of these a CU, the trees took 59 us.
// 32 rows a tile (RT = 2) at dims of 128 do not fit them, and take four waves: 8 x 8 rows of 32 heads on 8, 4000 keys, 43.5 us against 50 in two tiles of 16.
template <int NT, class C, int D, int RT, int NW>
__global__ __launch_bounds__(NW * 64, NW / 4) void paged_few_kernel(PagedAttentionArgs a, PagedPlan pl) {
    constexpr int QT = 16 * RT, G = 16 / sizeof(C), UK = 4 * G, HALVES = G / 8, NK = 2 * HALVES;   // NK: score tiles of a unit
    constexpr int KS = D / 32, KL = D / (4 * G), DT = D / 16, PT = NT == 1 && RT <= 2 ? 2 : NT;     // K-steps, loads a key row, output tiles, terms of a weight
    constexpr bool ROUNDED = PT == 1;                                 // weights have a divisor of their own
    __shared__ float o_s[NW][QT][D + 4], m_s[NW][QT], l_s[NW][QT], n_s[ROUNDED ? NW : 1][QT];
    __shared__ uint4 q_s[RT][KS][NT][64];                             // the queries as operands, alike for all waves
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int P = 1 << a.c.page_bits, group = pl.group;
    const size_t page_bytes = (size_t)a.c.n_kv * P * D * sizeof(C), head_bytes = (size_t)P * D * sizeof(C);
    const bool q_wide = (uintptr_t)a.q.p % 16 == 0 && (a.q.row | a.q.head) % 8 == 0, out_wide = (uintptr_t)a.out.p % 16 == 0 && (a.out.row | a.out.head) % 4 == 0;
    const PagedRuns<QT> runs(a, pl, kFewGroups, gridDim.x);
    const int w = blockIdx.x;
    if (w >= runs.n) return;
    unsigned pos = runs.start(w), before;
    const unsigned end = runs.start(w + 1);
    int s;
    runs.at(pos, s, before);
    PagedSeq<QT> seq;
    seq.init(a, pl, s, runs.flat);
    while (pos < end) {
        const unsigned off = pos - before, head_cost = seq.whole;
        if (off >= head_cost * a.c.n_kv) {                          // the next sequence with rows for this kernel
            before += head_cost * a.c.n_kv;
            if (s + 1 >= a.b.n_seqs) break;
            do seq.init(a, pl, ++s, runs.flat); while (seq.tiles == 0 && s + 1 < a.b.n_seqs);
            continue;
        }
        int h, t;
        unsigned first_cost;
        seq.at(off, a.c.n_kv, runs.flat, h, t, first_cost);
        const unsigned cost = seq.cost(t), x0 = off - first_cost, x1 = min(cost, x0 + (end - pos));
        // ---- the tile: packed rows t * QT .. , keys of all its rows
        const int packed = seq.n * group, valid = min(QT, packed - t * QT);
        const int i_first = t * QT / group, i_last = (t * QT + valid - 1) / group, len = seq.len;
        const int tile_end = a.seen ? min(len + min(seq.n, 64), a.b.capacity) : min(len + i_last + 1, a.b.capacity);
        const int tile_lo = a.window ? max(0, len + i_first - a.window + 1) / UK * UK : 0;
        const int units = tile_end > tile_lo ? (tile_end - tile_lo + UK - 1) / UK : 0;
        const int u0 = units_before(units, x0, cost), u1 = units_before(units, x1, cost);
        // a unit of keys all_lo .. all_hi - 1 is seen whole by every row
        const int all_hi = a.seen ? len : min(len + i_first + 1, a.b.capacity), all_lo = a.window ? max(0, len + i_last - a.window + 1) : 0;
        Sees sees[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int i = (min(16 * rt + r, valid - 1) + t * QT) / group;      // (rows behind the last: the last again)
            sees[rt].init(a, seq.first, len, i);
        }
        const float factor = a.scale * kLog2e * (sizeof(C) == 1 ? a.c.k_scale[h] : 1.0f);
        f32x4_t acc[RT][DT];
        float m[RT], l[RT], n[RT];                                  // maximum, sum of the weights, and as they are multiplied (ROUNDED)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = n[rt] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[rt][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        uint4 kf[NK][KL], vf[DT];
        int k_entry = 0, v_entry = 0, v_page = -1;                  // of the unit whose loads come next
        auto entries = [&](int u) {
            const int key = tile_lo + u * UK;
            k_entry = paged_entry(a.b, a.c, s, key + (r >> 2) * G);
            v_entry = paged_entry(a.b, a.c, s, key + g * G);
        };
        auto load_k = [&](int u) {
            const int at = tile_lo + u * UK + (r >> 2) * G, slot = (at & (P - 1)) + (r & 3), k_page = paged_entry_page(a.b, a.c, k_entry, at);
            const char *p = (const char *)a.c.k + (size_t)max(k_page, 0) * page_bytes + h * head_bytes + (size_t)(g * P + slot) * 16;
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int c = 0; c < KL; ++c) kf[n][c] = *reinterpret_cast<const uint4 *>(p + (size_t)c * 64 * P + n * 64);
        };
        auto load_v = [&](int u) {
            const int at = tile_lo + u * UK + g * G, slot = at & (P - 1);
            v_page = paged_entry_page(a.b, a.c, v_entry, at);
            const char *p = (const char *)a.c.v + (size_t)max(v_page, 0) * page_bytes + h * head_bytes + (size_t)(slot / G * D + r) * 16;
#pragma unroll
            for (int d = 0; d < DT; ++d) vf[d] = *reinterpret_cast<const uint4 *>(p + d * 256);
        };
        int u = u0 + wave;
        if (u < u1) {
            entries(u);
            load_k(u);
            load_v(u);
        }
        for (int x = wave; x < RT * KS; x += NW) {
            const int rt = x / KS, c = x % KS, pr = min(16 * rt + r, valid - 1) + t * QT, i = pr / group, j = pr - i * group;
            uint4 terms[NT];
            load_query<NT>(a, (size_t)(seq.first + i) * a.q.row + (size_t)(h * group + j) * a.q.head + (HALVES == 1 ? 32 * c + 8 * g : ((c / 2 * 4 + g) * 16 + c % 2 * 8)), q_wide, terms);
#pragma unroll
            for (int k = 0; k < NT; ++k) q_s[rt][c][k][lane] = terms[k];
        }
        __syncthreads();
        bool there = v_page >= 0;                                   // this lane's granule of the unit at hand
        if (u + NW < u1) entries(u + NW);
        for (; u < u1; u += NW) {
            const bool more = u + NW < u1;
            const int key0 = tile_lo + u * UK, key = key0 + g * G;   // key: of this lane's weights
            f32x4_t sc[RT][NK];
            asm volatile("" ::: "memory");                           // the queries are read again each time: as registers they leave room for too few waves
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) sc[rt][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                uint4 k[NK];
#pragma unroll
                for (int n = 0; n < NK; ++n) k[n] = operand<C>(kf[n][c / HALVES], c % HALVES);
#pragma unroll
                for (int i = NT - 1; i >= 0; --i)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const uint4 q = q_s[rt][c][i][lane];
#pragma unroll
                        for (int n = 0; n < NK; ++n) sc[rt][n] = mfma(k[n], q, sc[rt][n]);
                    }
            }
            if (more) load_k(u + NW);
            const bool whole = key0 >= all_lo && key0 + UK <= all_hi && __all(there);
            uint32_t seen_bits[RT];                                  // bit e: key + e
            bool odd_values = false;
            if (!whole) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    seen_bits[rt] = there ? sees[rt].keys(key, G, len, tile_end) : 0;
#pragma unroll
                    for (int e = 0; e < G; ++e) sc[rt][e / 4][e % 4] = seen_bits[rt] >> e & 1 ? sc[rt][e / 4][e % 4] : -INFINITY;
                }
                // values that nobody sees may be anything: zeros.  Others that are not finite are kept from the rows that do not see them (below).
                uint32_t bad = 0;
                uint32_t keep[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    constexpr int E = 4 / (int)sizeof(C);             // keys of a word
                    const int n = there ? min(max(tile_end - key - i * E, 0), E) : 0;
                    keep[i] = n == E ? 0xffffffffu : (1u << (8 * (int)sizeof(C) * n)) - 1;
                }
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    uint32_t *x = reinterpret_cast<uint32_t *>(&vf[d]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[i] &= keep[i];
                        if constexpr (sizeof(C) == 2) bad |= ((x[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                        else bad |= ((x[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                    }
                }
                odd_values = __any(bad != 0);
            }
            uint4 p[RT][HALVES][PT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float z[G], top = -INFINITY;
#pragma unroll
                for (int e = 0; e < G; ++e) {
                    z[e] = sc[rt][e / 4][e % 4] * factor;
                    if (!whole && !(seen_bits[rt] >> e & 1)) z[e] = -INFINITY;            // (a factor of 0 or below)
                    top = fmaxf(top, z[e]);
                }
                top = fmaxf(max_over_rows(top), m[rt]);
                const float use = top > -INFINITY ? top : 0.f;
                const float shrink = __builtin_amdgcn_exp2f(m[rt] - use);                // (0 at -infinity)
                m[rt] = top;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < G; ++e) {
                    z[e] = __builtin_amdgcn_exp2f(z[e] - use);
                    sum += z[e];
                }
                l[rt] = __builtin_fmaf(l[rt], shrink, sum);
                if constexpr (ROUNDED) n[rt] *= shrink;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[rt][d][i] *= shrink;
#pragma unroll
                for (int hv = 0; hv < HALVES; ++hv) {
                    uint32_t words[PT][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = z[8 * hv + 2 * i], y = z[8 * hv + 2 * i + 1];
#pragma unroll
                        for (int k = 0; k < PT; ++k) {
                            words[k][i] = two_bf16(x, y);
                            x -= bf16_lo(words[k][i]);
                            y -= bf16_hi(words[k][i]);
                        }
                        if constexpr (ROUNDED) n[rt] = add_two(words[0][i], n[rt]);
                    }
#pragma unroll
                    for (int k = 0; k < PT; ++k) p[rt][hv][k] = uint4{words[k][0], words[k][1], words[k][2], words[k][3]};
                }
            }
            if (!odd_values) {
#pragma unroll
                for (int d0 = 0; d0 < DT; d0 += 4)                    // four outputs at a time: a product does not wait for the one before it
#pragma unroll
                    for (int hv = 0; hv < HALVES; ++hv) {
                        uint4 v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = operand<C>(vf[d0 + i], hv);
#pragma unroll
                        for (int k = PT - 1; k >= 0; --k)
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[rt][d0 + i] = mfma(v[i], p[rt][hv][k], acc[rt][d0 + i]);
                    }
            } else {                                                 // one row at a time, with zeros where it does not see
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll 1
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t bits = __shfl(seen_bits[rt], 16 * g + j);
#pragma unroll
                        for (int hv = 0; hv < HALVES; ++hv) {
                            uint32_t keep[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) keep[i] = (bits >> (8 * hv + 2 * i) & 1 ? 0xffffu : 0u) | (bits >> (8 * hv + 2 * i) & 2 ? 0xffff0000u : 0u);
#pragma unroll
                            for (int d = 0; d < DT; ++d) {
                                uint4 raw = vf[d];                   // (widened here each time: as many registers again otherwise)
                                asm volatile("" : "+v"(raw.x), "+v"(raw.y), "+v"(raw.z), "+v"(raw.w));
                                uint4 v = operand<C>(raw, hv);
                                v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
                                f32x4_t one = acc[rt][d];            // (the other columns of the product are not theirs)
#pragma unroll
                                for (int k = PT - 1; k >= 0; --k) one = mfma(v, p[rt][hv][k], one);
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[rt][d][i] = r == j ? one[i] : acc[rt][d][i];
                            }
                        }
                    }
            }
            if (more) load_v(u + NW);
            there = v_page >= 0;
            if (u + 2 * NW < u1) entries(u + 2 * NW);
        }
        // ---- the waves' parts
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = xor_reduce<32, 16>(l[rt], AddOp());
            if constexpr (ROUNDED) n[rt] = xor_reduce<32, 16>(n[rt], AddOp());
            if (g == 0) {
                m_s[wave][16 * rt + r] = m[rt];
                l_s[wave][16 * rt + r] = l[rt];
                if constexpr (ROUNDED) n_s[wave][16 * rt + r] = n[rt];
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<float4 *>(&o_s[wave][16 * rt + r][16 * d + 4 * g]) = float4{acc[rt][d][0], acc[rt][d][1], acc[rt][d][2], acc[rt][d][3]};
        }
        __syncthreads();
        const bool alone = x0 == 0 && x1 == cost;
        const unsigned item = pos - x0;
        const int wa = alone ? w : runs.of(item), wb = alone ? w : runs.of(item + cost - 1);
        constexpr int kSlot = slot_floats(QT, D);
        float *slot = pl.slots + (size_t)(2 * w + (w == wa)) * kSlot;
        const float v_scale = sizeof(C) == 1 ? a.c.v_scale[h] : 1.0f;
        auto finish = [&](int row, int d, float top, float sum, float rounded, float (&o)[4]) {
            const int pr = t * QT + row, i = pr / group, j = pr - i * group;
            const bool empty = top == -INFINITY && sum == 0.f;
            const float by = empty ? 0.f : v_scale / (ROUNDED ? rounded : sum);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = empty ? 0.f : o[k] * by;
            store_output<NT>(a, (size_t)(seq.first + i) * a.out.row + (size_t)(h * group + j) * a.out.head + d, out_wide, o);
            if (a.lse && d == 0) a.lse[(size_t)(seq.first + i) * a.n_heads + h * group + j] = empty ? -INFINITY : (top + __log2f(sum)) * kLn2;
        };
        for (int idx = tid; idx < valid * (D / 4); idx += NW * 64) {
            const int row = idx / (D / 4), d = idx % (D / 4) * 4;
            float top = m_s[0][row], sum = 0.f, rounded = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 1; k < NW; ++k) top = fmaxf(top, m_s[k][row]);
            const float use = top > -INFINITY ? top : 0.f;
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float f = __builtin_amdgcn_exp2f(m_s[k][row] - use);
                const float4 x = *reinterpret_cast<const float4 *>(&o_s[k][row][d]);
                sum = __builtin_fmaf(l_s[k][row], f, sum);
                if constexpr (ROUNDED) rounded = __builtin_fmaf(n_s[k][row], f, rounded);
                o[0] = __builtin_fmaf(x.x, f, o[0]);
                o[1] = __builtin_fmaf(x.y, f, o[1]);
                o[2] = __builtin_fmaf(x.z, f, o[2]);
                o[3] = __builtin_fmaf(x.w, f, o[3]);
            }
            if (alone) {
                finish(row, d, top, sum, rounded, o);
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    __hip_atomic_store(reinterpret_cast<u64 *>(slot + row * D + d) + k, (u64)__float_as_uint(o[2 * k + 1]) << 32 | __float_as_uint(o[2 * k]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (d == 0) {
                    agent_store(slot + QT * D + row, top);
                    agent_store(slot + QT * D + QT + row, sum);
                    if constexpr (ROUNDED) agent_store(slot + QT * D + 2 * QT + row, rounded);
                }
            }
        }
        if (!alone) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // the part is acknowledged by memory
            __syncthreads();
            u64 *flag = pl.flags + 2 * w + (w == wa);
            if (tid == 0) {
                __hip_atomic_store(flag, pl.number, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            __syncthreads();
            bool all_there = true;
            for (int k = wa + tid; k <= wb; k += NW * 64)
                all_there &= __hip_atomic_load(pl.flags + 2 * k + (k == wa), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pl.number;
            if (__syncthreads_and(all_there)) {                     // (two may find so: they write the same)
                for (int idx = tid; idx < valid * (D / 4); idx += NW * 64) {
                    const int row = idx / (D / 4), d = idx % (D / 4) * 4;
                    float top = -INFINITY, sum = 0.f, rounded = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
                    constexpr int B = 4;                              // parts whose loads are on their way together
                    for (int k0 = wa; k0 <= wb; k0 += B) {
                        float pm[B], ps[B], pn[B];
                        u64 po[B][2];
#pragma unroll
                        for (int k = 0; k < B; ++k) {
                            const int from = min(k0 + k, wb);
                            const float *part = pl.slots + (size_t)(2 * from + (from == wa)) * kSlot;
                            pm[k] = agent_load(part + QT * D + row);
                            ps[k] = agent_load(part + QT * D + QT + row);
                            if constexpr (ROUNDED) pn[k] = agent_load(part + QT * D + 2 * QT + row);
#pragma unroll
                            for (int e = 0; e < 2; ++e) po[k][e] = __hip_atomic_load(reinterpret_cast<const u64 *>(part + row * D + d) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        }
#pragma unroll
                        for (int k = 0; k < B; ++k) {
                            const float x = k0 + k <= wb ? pm[k] : -INFINITY, higher = fmaxf(top, x), use = higher > -INFINITY ? higher : 0.f;
                            const float f = __builtin_amdgcn_exp2f(x - use), shrink = __builtin_amdgcn_exp2f(top - use);
                            top = higher;
                            if (k0 + k > wb) continue;
                            sum = __builtin_fmaf(ps[k], f, sum * shrink);
                            if constexpr (ROUNDED) rounded = __builtin_fmaf(pn[k], f, rounded * shrink);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(__uint_as_float((unsigned)(po[k][e / 2] >> (e % 2 * 32))), f, o[e] * shrink);
                        }
                    }
                    finish(row, d, top, sum, rounded, o);
                }
                for (int k = wa + tid; k <= wb; k += NW * 64)            // for the next call that carries this number (a replay)
                    __hip_atomic_store(pl.flags + 2 * k + (k == wa), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        __syncthreads();                                             // the next tile writes the waves' parts again
        pos += x1 - x0;
    }
}

// ---- many rows: the waves of a workgroup share tiles of 64 keys in LDS -----------------------------
// Each wave has 16 RT rows of the tile.  Keys and values come straight into LDS (e4m3: through registers, widened on the way) ahead of their use, in
// such an order that every operand of the matrix cores is 16 neighbouring granules: place 32 u + 16 n + r of a tile of keys holds key
// 32 u + 8 (r / 4) + 4 n + r % 4, the row r of score tile n of unit u.
//
// A prompt of 4096 rows, 32 heads on 8 of 128, bf16: 169 to 187 us, as the clock has it, 730 to 810 TFLOP/s (a large bf16 product of the library reaches 1242).  A SIMD's matrix
// core has a third of the cycles, other vector instructions about as much, and the two waves of a SIMD overlap them only in part; a tile's first loads and its results are
// about 10 us beside 33 steps of 1.6.  Steps, one after another: scores and weights in turn on one path 422 us; a loop of its own for steps seen whole (the registers
// of masks spilled in all) 261; the scores a step ahead, no maximum in between and operands read two groups ahead 255; tiles one by one instead of runs 188 (168 where the same
// was timed with others); the sum of the rounded weights, an instruction for two of them, 174 there.
// Tried: RT = 1, 201 us where RT = 2 takes 169; workgroups of eight waves, 166 there and 322 for 512 rows over 32000 keys (355), but 83 for 2 x 1351 rows of 32 heads (69);
// a load into LDS a group of products instead of all at once, 202 (193).  Pieces of 1 to 700 rows, 14 heads on 2 of 64, window 1000, float32: 43 us: 390 tiles in
// one round on 256 CUs, each a chain of 17 steps of 1.4 us behind the plan and first loads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ unsigned lds_place(const void *p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }
// 16 bytes a lane, from any address each, to 1 KiB from dst on
__device__ __forceinline__ void to_lds(const void *src, unsigned dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(dst)), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

template <int NT, class C, int D, int RT>
__global__ __launch_bounds__(256, 2) void paged_many_kernel(PagedAttentionArgs a, PagedPlan pl) {
    constexpr int QT = 64 * RT, G = 16 / sizeof(C), KT = 64, KS = D / 32, DT = D / 16, PT = NT;
    constexpr bool ROUNDED = PT == 1;                                 // weights have a divisor of their own
    constexpr bool WIDEN = sizeof(C) == 1;
    constexpr int LOADS = D / 8 * KT / 256;                          // granules of 16 bytes a thread brings of K, and of V (bf16)
    __shared__ uint4 k_s[2][D / 8][KT], v_s[2][KT / 8][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int P = 1 << a.c.page_bits, group = pl.group;
    const size_t page_bytes = (size_t)a.c.n_kv * P * D * sizeof(C), head_bytes = (size_t)P * D * sizeof(C);
    const bool q_wide = (uintptr_t)a.q.p % 16 == 0 && (a.q.row | a.q.head) % 8 == 0, out_wide = (uintptr_t)a.out.p % 16 == 0 && (a.out.row | a.out.head) % 4 == 0;
    const PagedRuns<QT> runs(a, pl, kGroups, gridDim.x);
    if ((int)blockIdx.x >= runs.n) return;
    // Workgroups on one XCD have neighbours in the row of tiles, which read the same keys; one by one the heads alternate, and with them the XCDs
    const int eighth = runs.n / 8, w = !runs.flat && (int)blockIdx.x < 8 * eighth ? (int)(blockIdx.x % 8 * eighth + blockIdx.x / 8) : (int)blockIdx.x;
    unsigned pos = runs.start(w), before;
    const unsigned end = runs.start(w + 1);
    int s;
    runs.at(pos, s, before);
    PagedSeq<QT> seq;
    seq.init(a, pl, s, runs.flat);
    const int my_key = (lane & 32) + ((lane & 15) >> 2) * 8 + (lane & 16 ? 4 : 0) + (lane & 3);        // the key of this lane's place
    while (pos < end) {
        const unsigned off = pos - before, head_cost = seq.whole;
        if (off >= head_cost * a.c.n_kv) {
            before += head_cost * a.c.n_kv;
            if (s + 1 >= a.b.n_seqs) break;
            do seq.init(a, pl, ++s, runs.flat); while (seq.tiles == 0 && s + 1 < a.b.n_seqs);
            continue;
        }
        int h, t;
        unsigned first_cost;
        seq.at(off, a.c.n_kv, runs.flat, h, t, first_cost);
        const unsigned cost = seq.cost(t), x0 = off - first_cost, x1 = min(cost, x0 + (end - pos));
        const int packed = seq.n * group, valid = min(QT, packed - t * QT), len = seq.len;
        const int i_first = t * QT / group, i_last = (t * QT + valid - 1) / group;
        const int tile_end = a.seen ? min(len + min(seq.n, 64), a.b.capacity) : min(len + i_last + 1, a.b.capacity);
        const int tile_lo = a.window ? max(0, len + i_first - a.window + 1) / KT * KT : 0;
        const int steps = tile_end > tile_lo ? (tile_end - tile_lo + KT - 1) / KT : 0;
        const int j0 = units_before(steps, x0, cost), j1 = units_before(steps, x1, cost);
        // this wave's rows
        const int row0 = wave * 16 * RT, rows = min(16 * RT, valid - row0);             // (0 or fewer: none)
        const int wi_first = (t * QT + min(row0, valid - 1)) / group, wi_last = (t * QT + max(0, min(row0 + 16 * RT, valid) - 1)) / group;
        const int all_hi = a.seen ? len : min(len + wi_first + 1, a.b.capacity), all_lo = a.window ? max(0, len + wi_last - a.window + 1) : 0;
        const int any_hi = a.seen ? tile_end : min(len + wi_last + 1, a.b.capacity), any_lo = a.window ? max(0, len + wi_first - a.window + 1) : 0;
        uint4 q[RT][KS][NT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int pr = min(row0 + 16 * rt + r, valid - 1) + t * QT, i = pr / group, j = pr - i * group;
            const size_t at = (size_t)(seq.first + i) * a.q.row + (size_t)(h * group + j) * a.q.head;
#pragma unroll
            for (int c = 0; c < KS; ++c) load_query<NT>(a, at + 32 * c + 8 * g, q_wide, q[rt][c]);
            if (a.scale < 0.f) {
#pragma unroll
                for (int c = 0; c < KS; ++c)
#pragma unroll
                    for (int i2 = 0; i2 < NT; ++i2) {
                        uint4 &x = q[rt][c][i2];
                        x.x ^= 0x80008000u; x.y ^= 0x80008000u; x.z ^= 0x80008000u; x.w ^= 0x80008000u;
                    }
            }
        }
        const float factor = fmaxf(fabsf(a.scale) * kLog2e * (WIDEN ? a.c.k_scale[h] : 1.0f), __FLT_DENORM_MIN__);       // (0: positions that are not seen stay at -infinity)
        f32x4_t acc[RT][DT];
        float m[RT], l[RT], n[RT];                                  // maximum, sum of the weights, and as they are multiplied (ROUNDED)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = n[rt] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[rt][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        // Entries of the page table for the steps whose loads come next: of this lane's key, and of the granules of values that this wave (e4m3: thread) brings.
        // Keys behind the tile's last are nobody's: their place need not exist.
        constexpr int VG = WIDEN ? (D == 128 ? 2 : 1) : 2;
        int k_entry = 0, v_entry[VG];
        auto v_granule = [&](int i) { return WIDEN ? (tid + 256 * i) / D * 2 : wave * 2 + i; };        // of 8 keys
        auto k_at = [&](int j) { return tile_lo + j * KT + my_key; };
        auto v_at = [&](int j, int i) { return tile_lo + j * KT + v_granule(i) * 8; };
        auto page_of = [&](int entry, int key) { return key < tile_end ? paged_entry_page(a.b, a.c, entry, key) : 0; };
        auto page_at = [&](int key) { return page_of(paged_entry(a.b, a.c, s, key), key); };
        auto v_entries = [&](int j, int (&to)[VG]) {
#pragma unroll
            for (int i = 0; i < VG; ++i) to[i] = paged_entry(a.b, a.c, s, v_at(j, i));
        };
        auto k_entries = [&](int j) { return paged_entry(a.b, a.c, s, k_at(j)); };
        uint4 kr[WIDEN ? LOADS / 2 : 1], vr[WIDEN ? LOADS / 2 : 1];
        bool k_there = true;                                         // whether all keys of the step loaded last have a place
        auto load_k = [&](int j) {
            const int key = tile_lo + j * KT, buf = j & 1, page = page_of(k_entry, k_at(j));
            k_there = __all(page >= 0);
            const char *kp = (const char *)a.c.k + (size_t)max(page, 0) * page_bytes + h * head_bytes + (size_t)((key + my_key) & (P - 1)) * 16;
            if constexpr (WIDEN) {
#pragma unroll
                for (int i = 0; i < LOADS / 2; ++i) kr[i] = *reinterpret_cast<const uint4 *>(kp + (size_t)(wave + 4 * i) * P * 16);
            } else {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) to_lds(kp + (size_t)(wave * (D / 32) + i) * P * 16, lds_place(&k_s[buf][wave * (D / 32) + i][0]));
            }
        };
        auto load_v = [&](int j) {
            const int key = tile_lo + j * KT, buf = j & 1;
            if constexpr (WIDEN) {
#pragma unroll
                for (int i = 0; i < LOADS / 2; ++i) {
                    const int d = (tid + 256 * i) % D, slot = (key + v_granule(i) * 8) & (P - 1);
                    vr[i] = *reinterpret_cast<const uint4 *>((const char *)a.c.v + (size_t)max(page_of(v_entry[i], v_at(j, i)), 0) * page_bytes + h * head_bytes + (size_t)(slot / G * D + d) * 16);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int slot = (key + v_granule(i) * 8) & (P - 1);
                    const char *vp = (const char *)a.c.v + (size_t)max(page_of(v_entry[i], v_at(j, i)), 0) * page_bytes + h * head_bytes + (size_t)(slot / G * D + lane) * 16;
#pragma unroll
                    for (int x = 0; x < D / 64; ++x) to_lds(vp + x * 1024, lds_place(&v_s[buf][wave * 2 + i][64 * x]));
                }
            }
        };
        auto widen_k = [&](int j) {
            if constexpr (WIDEN) {
#pragma unroll
                for (int i = 0; i < LOADS / 2; ++i) {
                    const int c = wave + 4 * i;
                    k_s[j & 1][2 * c][lane] = operand<C>(kr[i], 0);
                    k_s[j & 1][2 * c + 1][lane] = operand<C>(kr[i], 1);
                }
            }
        };
        auto widen_v = [&](int j) {
            if constexpr (WIDEN) {
#pragma unroll
                for (int i = 0; i < LOADS / 2; ++i) {
                    const int d = (tid + 256 * i) % D, gv = v_granule(i);
                    v_s[j & 1][gv][d] = operand<C>(vr[i], 0);
                    v_s[j & 1][gv + 1][d] = operand<C>(vr[i], 1);
                }
            }
        };
        // The scores of step j + 1 are multiplied while the weights of step j are made, so keys are brought two steps ahead, values one.
        bool there = true, there_next = true;                        // whether all keys of steps j and j + 1 have a place
        f32x4_t sc[RT][4];
        auto scores = [&](int j, f32x4_t (&x)[RT][4]) {
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) x[rt][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                uint4 kf[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) kf[n] = k_s[j & 1][c * 4 + g][16 * n + r];
#pragma unroll
                for (int i = NT - 1; i >= 0; --i)
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) x[rt][n] = mfma(kf[n], q[rt][c][i], x[rt][n]);
            }
        };
        auto arrived = [] {                                          // this wave's loads are in LDS and its reads done, then everybody's
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __syncthreads();
        };
        if (j0 < j1) {
            // all entries that the first steps need on their way at once, with the queries; then the keys and values
            int v_next[VG];
            k_entry = k_entries(j0);
            const int k_second = k_entries(min(j0 + 1, j1 - 1)), k_third = k_entries(min(j0 + 2, j1 - 1));
            v_entries(j0, v_entry);
            v_entries(min(j0 + 1, j1 - 1), v_next);
            int k_next = k_second, k_after = k_third;
            asm volatile("" : "+v"(k_entry), "+v"(k_next), "+v"(k_after));
#pragma unroll
            for (int i = 0; i < VG; ++i) asm volatile("" : "+v"(v_entry[i]), "+v"(v_next[i]));
            load_k(j0);
            there = k_there;
            load_v(j0);
            widen_k(j0);
            widen_v(j0);
            if (j0 + 1 < j1) {
                k_entry = k_next;
                load_k(j0 + 1);
                there_next = k_there;
                widen_k(j0 + 1);
            }
            k_entry = k_after;
#pragma unroll
            for (int i = 0; i < VG; ++i) v_entry[i] = v_next[i];
            // The queries have to be there before the loop: the compiler does not count the loads into LDS, and a wait for the queries inside it would be one
            // for those loads.
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int c = 0; c < KS; ++c)
#pragma unroll
                    for (int k = 0; k < NT; ++k) asm volatile("" : "+v"(q[rt][c][k].x), "+v"(q[rt][c][k].y), "+v"(q[rt][c][k].z), "+v"(q[rt][c][k].w));
            arrived();
            scores(j0, sc);
        }
        bool there_after = true;
        auto enter = [&](int j) {                                    // step j's values and step j + 1's keys are in LDS after this
            arrived();
            // the entries are there as well, and have to be so for the compiler: its wait for them behind the loads below would be one for those
            asm volatile("" : "+v"(k_entry));
#pragma unroll
            for (int i = 0; i < VG; ++i) asm volatile("" : "+v"(v_entry[i]));
            if (j + 2 < j1) {
                load_k(j + 2);
                there_after = k_there;
            }
            if (j + 1 < j1) load_v(j + 1);
            if (j + 3 < j1) k_entry = k_entries(j + 3);
            if (j + 2 < j1) v_entries(j + 2, v_entry);
        };
        auto leave = [&](int j) {
            if (j + 2 < j1) widen_k(j + 2);
            if (j + 1 < j1) widen_v(j + 1);
            there = there_next;
            there_next = there_after;
        };
        auto whole_at = [&](int j) { return there && tile_lo + j * KT >= all_lo && tile_lo + j * KT + KT <= all_hi && rows > 0; };
        auto step = [&](auto whole_, const int j) {
            constexpr bool WHOLE = decltype(whole_)::value;
            const int key0 = tile_lo + j * KT, buf = j & 1;
            f32x4_t next[RT][4];                                      // (behind the last step: of whatever is there, for nobody)
            if constexpr (!WHOLE) scores(j + 1, next);
            {
                uint32_t seen_bits[RT];                               // bit 8 u + e: key 32 u + 8 g + e of the step
                if constexpr (!WHOLE) {
                    bool here[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) here[u] = there || page_at(key0 + 32 * u + 8 * g) >= 0;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        Sees sees;
                        sees.init(a, seq.first, len, (min(row0 + 16 * rt + r, valid - 1) + t * QT) / group);
                        seen_bits[rt] = 0;
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            if (here[u]) seen_bits[rt] |= sees.keys(key0 + 32 * u + 8 * g, 8, len, tile_end) << (8 * u);
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sc[rt][n][i] = seen_bits[rt] >> (4 * n + i) & 1 ? sc[rt][n][i] : -INFINITY;
                    }
                }
                // Weights: exponentials above a row's reference, which is the maximum at the time it was set.  It is set again only where a lane's sum
                // passes 2^10 (or nothing was seen before): the steps in between need no maximum.
                uint4 p[RT][2][PT];
                float sum[RT], rounded[RT];
                // half a row tile's: 32 keys
                auto weights = [&](int rt, int u) {
                    const float use = m[rt] > -INFINITY ? m[rt] : 0.f;
                    if (u == 0) sum[rt] = rounded[rt] = 0.f;
                    uint32_t words[PT][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4_t &z = sc[rt][2 * u + i / 2];
                        float x = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i % 2 * 2], factor, -use)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i % 2 * 2 + 1], factor, -use));
                        sum[rt] += x;
                        sum[rt] += y;
#pragma unroll
                        for (int k = 0; k < PT; ++k) {
                            words[k][i] = two_bf16(x, y);
                            if (k + 1 < PT) {
                                x -= bf16_lo(words[k][i]);
                                y -= bf16_hi(words[k][i]);
                            }
                        }
                        if constexpr (ROUNDED) rounded[rt] = add_two(words[0][i], rounded[rt]);
                    }
#pragma unroll
                    for (int k = 0; k < PT; ++k) p[rt][u][k] = uint4{words[k][0], words[k][1], words[k][2], words[k][3]};
                };
                // The operands in LDS are read two groups of products ahead, and the order is held: left to itself the compiler reads each just
                // before its use, and the wave waits for LDS at every second product.
                constexpr int VB = 4, NB = 2 * DT / VB;               // operands a group, groups of the second product
                uint4 vb[2][VB];
                auto read_v = [&](int x) {
#pragma unroll
                    for (int i = 0; i < VB; ++i) vb[x & 1][i] = v_s[buf][4 * ((x * VB + i) / DT) + g][16 * ((x * VB + i) % DT) + r];
                };
                if constexpr (WHOLE) {
                    uint4 kf[2][4];
                    auto read_k = [&](int c) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) kf[c & 1][n] = k_s[(j + 1) & 1][c * 4 + g][16 * n + r];
                    };
                    read_k(0);
                    read_k(1);
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) next[rt][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < KS; ++c) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int i = NT - 1; i >= 0; --i)
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int rt = 0; rt < RT; ++rt) next[rt][n] = mfma(kf[c & 1][n], q[rt][c][i], next[rt][n]);
                        if (c + 2 < KS) read_k(c + 2);
                        else read_v(c + 2 - KS);
#pragma unroll
                        for (int x = c * 2 * RT / KS; x < (c + 1) * 2 * RT / KS; ++x) weights(x / 2, x % 2);
#pragma unroll
                        for (int i = 0; i < 4 * RT * NT; ++i) {       // in turn
                            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                            __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                } else {
#pragma unroll
                    for (int x = 0; x < 2 * RT; ++x) weights(x / 2, x % 2);
                }
                bool set = false;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) set |= sum[rt] > 1024.f || m[rt] == -INFINITY;
                if (__any(set)) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        float top = -INFINITY;
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[rt][n][i]);
                        top = max_over_rows(top) * factor;
                        const bool mine = max_over_rows(sum[rt]) > 1024.f || m[rt] == -INFINITY;      // (a row's result does not depend on the others')
                        top = mine ? fmaxf(top, m[rt]) : m[rt];
                        const float shrink = __builtin_amdgcn_exp2f(m[rt] - (top > -INFINITY ? top : 0.f));
                        m[rt] = top;
                        l[rt] *= shrink;
                        if constexpr (ROUNDED) n[rt] *= shrink;
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[rt][d][i] *= shrink;
                        weights(rt, 0);
                        weights(rt, 1);
                    }
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    l[rt] += sum[rt];
                    if constexpr (ROUNDED) n[rt] += rounded[rt];
                }
                if constexpr (WHOLE) {
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int k = PT - 1; k >= 0; --k)             // (terms outside: a product does not wait for the one before it)
#pragma unroll
                            for (int i = 0; i < VB; ++i)
#pragma unroll
                                for (int rt = 0; rt < RT; ++rt) {
                                    const int d = (x * VB + i) % DT, u = (x * VB + i) / DT;
                                    acc[rt][d] = mfma(vb[x & 1][i], p[rt][u][k], acc[rt][d]);
                                }
                        if (x + 2 < NB) read_v(x + 2);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    // values of places that do not exist may be anything: zeros; others that are not finite are kept from the rows that do not see them
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int key = key0 + 32 * u + 8 * g;
                        const bool here = there || page_at(key) >= 0;
                        uint32_t keep[4], bad = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int n = here ? min(max(tile_end - key - 2 * i, 0), 2) : 0;
                            keep[i] = n == 2 ? 0xffffffffu : (1u << (16 * n)) - 1;
                        }
                        auto value = [&](int d) {
                            uint4 v = v_s[buf][4 * u + g][16 * d + r];
                            v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
                            return v;
                        };
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const uint4 v = value(d);
                            bad |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) | ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
                        }
                        const bool finite = !__any((bad & 0x80008000u) != 0);
                        asm volatile("" ::: "memory");
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            if (finite) {
#pragma unroll
                                for (int d = 0; d < DT; ++d) {
                                    const uint4 v = value(d);
#pragma unroll
                                    for (int k = PT - 1; k >= 0; --k) acc[rt][d] = mfma(v, p[rt][u][k], acc[rt][d]);
                                }
                            } else {
#pragma unroll 1
                                for (int x = 0; x < 16; ++x) {               // one row at a time, with zeros where it does not see
                                    asm volatile("" ::: "memory");
                                    const uint32_t bits = (uint32_t)__shfl((int)seen_bits[rt], 16 * g + x) >> (8 * u);
                                    uint32_t mine[4];
#pragma unroll
                                    for (int i = 0; i < 4; ++i) mine[i] = (bits >> (2 * i) & 1 ? 0xffffu : 0u) | (bits >> (2 * i) & 2 ? 0xffff0000u : 0u);
#pragma unroll
                                    for (int d = 0; d < DT; ++d) {
                                        uint4 v = value(d);
                                        v.x &= mine[0]; v.y &= mine[1]; v.z &= mine[2]; v.w &= mine[3];
                                        f32x4_t one = acc[rt][d];
#pragma unroll
                                        for (int k = PT - 1; k >= 0; --k) one = mfma(v, p[rt][u][k], one);
#pragma unroll
                                        for (int i = 0; i < 4; ++i) acc[rt][d][i] = r == x ? one[i] : acc[rt][d][i];
                                    }
                                }
                            }
                        }
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) sc[rt][n] = next[rt][n];
        };
        // (a loop of its own for the steps that every row of the wave sees whole: one loop with both kinds spills in both)
        for (int j = j0; j < j1;) {
            for (; j < j1 && whole_at(j); ++j) {
                enter(j);
                step(std::integral_constant<bool, true>(), j);
                leave(j);
            }
            for (; j < j1 && !whole_at(j); ++j) {
                const int key0 = tile_lo + j * KT;
                enter(j);
                if (rows > 0 && key0 < any_hi && key0 + KT > any_lo) step(std::integral_constant<bool, false>(), j);
                else scores(j + 1, sc);
                leave(j);
            }
        }
        __syncthreads();                                              // the next tile's loads write what other waves may still read
        // ---- results
        const bool alone = x0 == 0 && x1 == cost;
        const unsigned item = pos - x0;
        const int wa = alone ? w : runs.of(item), wb = alone ? w : runs.of(item + cost - 1);
        constexpr int kSlot = slot_floats(QT, D);
        float *slot = pl.slots + (size_t)(2 * w + (w == wa)) * kSlot;
        const float v_scale = WIDEN ? a.c.v_scale[h] : 1.0f;
        auto finish = [&](int rt) {
            if (16 * rt + r >= rows) return;
            const int pr = t * QT + row0 + 16 * rt + r, i = pr / group, j = pr - i * group;
            const bool empty = m[rt] == -INFINITY && l[rt] == 0.f;
            const float by = empty ? 0.f : v_scale / (ROUNDED ? n[rt] : l[rt]);
            const size_t at = (size_t)(seq.first + i) * a.out.row + (size_t)(h * group + j) * a.out.head + 4 * g;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                float o[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) o[k] = empty ? 0.f : acc[rt][d][k] * by;
                store_output<NT>(a, at + 16 * d, out_wide, o);
            }
            if (a.lse && g == 0) a.lse[(size_t)(seq.first + i) * a.n_heads + h * group + j] = empty ? -INFINITY : (m[rt] + __log2f(l[rt])) * kLn2;
        };
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = xor_reduce<32, 16>(l[rt], AddOp());
            if constexpr (ROUNDED) n[rt] = xor_reduce<32, 16>(n[rt], AddOp());
            if (alone) {
                finish(rt);
            } else if (16 * rt + r < rows) {
                const int row = row0 + 16 * rt + r;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        const u64 two = (u64)__float_as_uint(acc[rt][d][k + 1]) << 32 | __float_as_uint(acc[rt][d][k]);
                        __hip_atomic_store(reinterpret_cast<u64 *>(slot + row * D + 16 * d + 4 * g + k), two, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                if (g == 0) {
                    agent_store(slot + QT * D + row, m[rt]);
                    agent_store(slot + QT * D + QT + row, l[rt]);
                    if constexpr (ROUNDED) agent_store(slot + QT * D + 2 * QT + row, n[rt]);
                }
            }
        }
        if (!alone) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) {
                __hip_atomic_store(pl.flags + 2 * w + (w == wa), pl.number, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            __syncthreads();
            bool all_there = true;
            for (int k = wa + tid; k <= wb; k += 256)
                all_there &= __hip_atomic_load(pl.flags + 2 * k + (k == wa), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pl.number;
            if (__syncthreads_and(all_there)) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if (16 * rt + r >= rows) continue;
                    const int row = row0 + 16 * rt + r;
                    float top = -INFINITY, sum = 0.f, rounded = 0.f;
                    for (int k = wa; k <= wb; ++k) top = fmaxf(top, agent_load(pl.slots + (size_t)(2 * k + (k == wa)) * kSlot + QT * D + row));
                    const float use = top > -INFINITY ? top : 0.f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) acc[rt][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    for (int k = wa; k <= wb; ++k) {
                        const float *part = pl.slots + (size_t)(2 * k + (k == wa)) * kSlot;
                        const float f = __builtin_amdgcn_exp2f(agent_load(part + QT * D + row) - use);
                        sum = __builtin_fmaf(agent_load(part + QT * D + QT + row), f, sum);
                        if constexpr (ROUNDED) rounded = __builtin_fmaf(agent_load(part + QT * D + 2 * QT + row), f, rounded);
                        u64 x[DT][2];
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                x[d][e] = __hip_atomic_load(reinterpret_cast<const u64 *>(part + row * D + 16 * d + 4 * g + 2 * e), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                acc[rt][d][2 * e] = __builtin_fmaf(__uint_as_float((unsigned)x[d][e]), f, acc[rt][d][2 * e]);
                                acc[rt][d][2 * e + 1] = __builtin_fmaf(__uint_as_float((unsigned)(x[d][e] >> 32)), f, acc[rt][d][2 * e + 1]);
                            }
                    }
                    m[rt] = top;
                    l[rt] = sum;
                    n[rt] = rounded;
                    finish(rt);
                }
                for (int k = wa + tid; k <= wb; k += 256) __hip_atomic_store(pl.flags + 2 * k + (k == wa), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        pos += x1 - x0;
    }
}

// ---- launches -----------------------------------------------------------------------

// Which kernel takes what, by packed rows.  Up to a mean of kFewMean a sequence the kernel of few rows, but for sequences of more than kFewMost, which the
// kernel of many rows takes in a launch of its own (not needed if there can be none); beyond that mean the kernel of many rows takes all.  As it is / few alone /
// many alone, us: 16 x 16 rows, 4 heads a key head, 4000 keys (mean 64) 96 / 92 / 122; 33 x 1 to 20, 500 to 8000 keys (42) 178 / 175 / 172; 64 x 1 to 4
// (10) 209 / 203 / 258; 8 x 8 (32) 45 / 44 / 85; pieces of prompts of up to 700 rows (2450) 42 / 71 / 41; 17 x 1 to 481, short (241) 53 / 148 / 53.
constexpr int kFewMean = 64, kFewMost = 256;
// row tiles of a wave of the kernel of many rows
constexpr int many_tiles(int NT, int held, int D) { return NT == 3 || (held == 1 && D == 128) ? 1 : 2; }

// Rows of a sequence at most: all, or, as long as no sequence is without any, all but one of each other.  What that says chooses kernels; one that is
// alone takes every sequence.
struct Kernels { int mean; bool few, many; };
static Kernels paged_kernels(const PagedBatchArgs &b, int group) {
    const int most = b.row_start ? std::max(1, b.n_rows - b.n_seqs + 1) : b.each, mean = (b.n_rows + b.n_seqs - 1) / b.n_seqs * group;
    const bool few = mean <= kFewMean;
    return {mean, few, !few || most * group > kFewMost};
}
// flags, slots, a head of zeros
static size_t zeros_at(bool many, int dim) { return 2 * kGroups * sizeof(u64) + 2 * (size_t)(many ? kGroups * slot_floats(128, dim) : kFewGroups * slot_floats(64, dim)) * sizeof(float); }
size_t paged_attention_workspace_bytes(const PagedCacheArgs &c, const PagedBatchArgs &b, int n_heads) {
    return zeros_at(paged_kernels(b, n_heads / c.n_kv).many, c.dim) + c.dim * sizeof(float);
}

// A number that no workspace holds by chance, another one each call
static u64 call_number() {
    static std::atomic<u64> calls{(u64)(uintptr_t)&calls * 0x9e3779b97f4a7c15ull};
    u64 x = calls.fetch_add(0x9e3779b97f4a7c15ull);
    x = (x ^ (x >> 30)) * 0xbf58476d1ce4e5b9ull;
    x = (x ^ (x >> 27)) * 0x94d049bb133111ebull;
    x ^= x >> 31;
    return x ? x : 1;
}

hipError_t launch_paged_attention(const PagedAttentionArgs &args, hipStream_t stream) {
    PagedAttentionArgs a = args;
    PagedPlan pl;
    pl.number = call_number();
    pl.group = a.n_heads / a.c.n_kv;
    pl.flags = (u64 *)a.workspace;
    pl.slots = (float *)(pl.flags + 2 * kGroups);
    const Kernels use = paged_kernels(a.b, pl.group);
    const int mean = use.mean;
    const bool few = use.few, both = use.few && use.many;
    if (a.scale == 0.f) {                  // all queries are one head of zeros: a product beyond float32's range would have no 0 to become
        a.q = {(char *)a.workspace + zeros_at(use.many, a.c.dim), 0, 0};
        const hipError_t rc = launch_fill_zero(a.q.p, a.c.dim * sizeof(float), stream);
        if (rc != hipSuccess) return rc;
    }
    // costs in 31 bits: the tiles of all heads, each of no more than this many keys
    // keys: what a workgroup takes at least (of sixteen batches none is more than 5 % off with half or twice as many).  join: what sharing costs, in keys: with 350 the pieces of
    // prompts (above) took 56 us, with 1024 47; with half of what stands below one token of 640 keys takes 16.5 us (11), 17 short prompts 71 (53); with twice as much 16 x 16
    // rows over 4000 keys 115 (96).
    auto costs = [&](int QT, int keys, int join) {
        const u64 tiles = ((u64)a.b.n_rows * pl.group / QT + a.b.n_seqs) * a.c.n_kv, span = (u64)a.b.capacity + (u64)a.b.n_rows * (pl.group / QT + 1) + 2 * QT + 256;
        pl.shift = 0;
        while (tiles * ((span >> pl.shift) + 2) >> 31) ++pl.shift;
        pl.least = std::max(1, keys >> pl.shift);
        pl.join = std::max(1, join >> pl.shift);
    };
    // as many workgroups as there can be tiles, so that each may be taken by one
    auto tiles_grid = [&](int QT, u64 least) { return (unsigned)std::min<u64>(std::max(least, ((u64)a.b.n_rows * pl.group / QT + a.b.n_seqs) * a.c.n_kv), 1 << 20); };
#define SPD_FEW(NT, C, D, RT, NW)                                                                                            \
    do {                                                                                                                     \
        costs(16 * RT, 512, 1100);                                                                                                 \
        hipLaunchKernelGGL((paged_few_kernel<NT, C, D, RT, NW>), dim3(tiles_grid(16 * RT, kFewGroups)), dim3(NW * 64), 0, stream, a, pl);                \
    } while (0)
#define SPD_FEW_RT(NT, C, D)                                                                                                 \
    do {                                                                                                                     \
        if (few) {                                                                                                           \
            pl.above = 0; pl.upto = both ? kFewMost : 0x7fffffff;                                                            \
            if (mean <= 16) SPD_FEW(NT, C, D, 1, 8);                                                                         \
            else if (mean <= 32 || NT == 3) SPD_FEW(NT, C, D, 2, (D == 64 ? 8 : 4));                                         \
            else SPD_FEW(NT, C, D, (NT == 3 ? 2 : 4), (NT == 3 && D == 64 ? 8 : 4));                                         \
        }                                                                                                                    \
        if (!few || both) {                                                                                                  \
            constexpr int RT = many_tiles(NT, sizeof(C), D);                                                                 \
            pl.above = few ? kFewMost : 0; pl.upto = 0x7fffffff;                                                             \
            costs(64 * RT, 512, 1024);                                                                                       \
            hipLaunchKernelGGL((paged_many_kernel<NT, C, D, RT>), dim3(tiles_grid(64 * RT, kGroups)), dim3(256), 0, stream, a, pl); \
        }                                                                                                                    \
    } while (0)
#define SPD_FEW_D(NT, C) do { if (a.c.dim == 64) SPD_FEW_RT(NT, C, 64); else SPD_FEW_RT(NT, C, 128); } while (0)
    if (a.bf16 && a.c.e4m3) SPD_FEW_D(1, uint8_t);
    else if (a.bf16) SPD_FEW_D(1, uint16_t);
    else if (a.c.e4m3) SPD_FEW_D(3, uint8_t);
    else SPD_FEW_D(3, uint16_t);
    return hipGetLastError();
}

}  // namespace spd
