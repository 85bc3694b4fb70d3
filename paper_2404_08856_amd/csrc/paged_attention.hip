// Attention of the new rows of sequences over their pages, on the matrix cores.
//
//   scores   S[key, row] = sum_d K[key, d] q[row, d]      v_mfma_f32_16x16x32_bf16, A = 16 keys x 32 dims, B = q
//   softmax  running maximum and sum per row, in base 2
//   output   O[d, row] = sum_key V[key, d] p[row, key]    A = 16 dims x 32 keys, B = p
//
// float32 rows: q and p as three bf16 terms each, exact to float32's roundings.  e4m3 keys and values are bf16 values, their scales one factor
// of a head's scores and of its output.  The rows of the score tiles are keys in such an order that a lane ends with the weights of a whole granule
// of keys, the 16 bytes of V that it reads for the second product: no data moves between lanes, and every load is 16 bytes of one granule.
#include <atomic>

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

constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;

// 8 neighbouring elements of a query as bf16 terms; flip: the sign bits to turn
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
// A wave takes units of four granules of keys (32 in bf16, 64 in e4m3), one in four of the workgroup's run.  The registers of K and V are filled again for the
// wave's next unit as soon as the product has read them.
template <int NT, class C, int D, int RT>
__global__ __launch_bounds__(256, RT == 1 ? 2 : 1) void paged_few_kernel(PagedAttentionArgs a, PagedPlan pl) {
    constexpr int QT = 16 * RT, G = 16 / sizeof(C), UK = 4 * G, HALVES = G / 8, NK = 2 * HALVES;   // NK: score tiles of a unit
    constexpr int KS = D / 32, KL = D / (4 * G), DT = D / 16, PT = NT == 1 ? 2 : 3;                 // K-steps, loads a key row, output tiles, terms of a weight
    __shared__ float o_s[4][QT][D + 4], m_s[4][QT], l_s[4][QT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int P = 1 << a.c.page_bits, group = pl.group;
    const size_t page_bytes = (size_t)a.c.n_kv * P * D * sizeof(C), head_bytes = (size_t)P * D * sizeof(C);
    const bool q_wide = (uintptr_t)a.q.p % 16 == 0 && (a.q.row | a.q.head) % 8 == 0, out_wide = (uintptr_t)a.out.p % 16 == 0 && (a.out.row | a.out.head) % 4 == 0;
    const PagedMap<QT> map(a, pl);
    PagedRuns runs;
    u64 mine;
    const u64 all = map.total(mine);
    if (all == 0) return;
    runs.init(all, pl.least, gridDim.x);
    const int w = blockIdx.x;
    if (w >= runs.n) return;
    u64 pos = runs.start(w), before;
    const u64 end = runs.start(w + 1);
    int s;
    map.at(pos, mine, s, before);
    PagedSeq<QT> seq;
    seq.init(a, pl, s);
    while (pos < end) {
        const u64 off = pos - before, head_cost = seq.before(seq.tiles);
        if (off >= head_cost * a.c.n_kv) {                          // the next sequence with rows for this kernel
            before += head_cost * a.c.n_kv;
            do seq.init(a, pl, ++s); while (seq.tiles == 0 && s + 1 < a.b.n_seqs);
            continue;
        }
        const int h = (int)(off / head_cost);
        const u64 in_head = off - h * head_cost;
        const int t = seq.tile_at(in_head);
        const u64 cost = seq.cost(t), x0 = in_head - seq.before(t), x1 = min(cost, x0 + (end - pos));
        // ---- the tile: packed rows t * QT .. , keys of all its rows
        const int packed = seq.n * group, valid = min(QT, packed - t * QT);
        const int i_first = t * QT / group, i_last = (t * QT + valid - 1) / group, len = seq.len;
        const int tile_end = a.seen ? min(len + min(seq.n, 64), a.b.capacity) : min(len + i_last + 1, a.b.capacity);
        const int tile_lo = a.window ? max(0, len + i_first - a.window + 1) / UK * UK : 0;
        const int units = tile_end > tile_lo ? (tile_end - tile_lo + UK - 1) / UK : 0;
        const int u0 = (int)((u64)units * x0 / cost), u1 = (int)((u64)units * x1 / cost);
        // a unit of keys all_lo .. all_hi - 1 is seen whole by every row
        const int all_hi = a.seen ? len : min(len + i_first + 1, a.b.capacity), all_lo = a.window ? max(0, len + i_last - a.window + 1) : 0;
        uint4 q[RT][KS][NT];
        Sees sees[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int pr = min(16 * rt + r, valid - 1) + t * QT, i = pr / group, j = pr - i * group;      // (rows behind the last: the last again)
            sees[rt].init(a, seq.first, len, i);
            const size_t at = (size_t)(seq.first + i) * a.q.row + (size_t)(h * group + j) * a.q.head;
#pragma unroll
            for (int c = 0; c < KS; ++c) load_query<NT>(a, at + (HALVES == 1 ? 32 * c + 8 * g : ((c / 2 * 4 + g) * 16 + c % 2 * 8)), q_wide, q[rt][c]);
        }
        const float factor = a.scale * kLog2e * (sizeof(C) == 1 ? a.c.k_scale[h] : 1.0f);
        f32x4_t acc[RT][DT];
        float m[RT], l[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[rt][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        uint4 kf[NK][KL], vf[DT];
        int k_page = -1, v_page = -1;                               // of the unit whose loads come next
        auto pages = [&](int u) {
            const int key = tile_lo + u * UK;
            k_page = paged_page(a.b, a.c, s, (key + (r >> 2) * G) >> a.c.page_bits);
            v_page = paged_page(a.b, a.c, s, (key + g * G) >> a.c.page_bits);
        };
        auto load_k = [&](int u) {
            const int slot = ((tile_lo + u * UK + (r >> 2) * G) & (P - 1)) + (r & 3);
            const char *p = (const char *)a.c.k + (size_t)max(k_page, 0) * page_bytes + h * head_bytes + (size_t)(g * P + slot) * 16;
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int c = 0; c < KL; ++c) kf[n][c] = *reinterpret_cast<const uint4 *>(p + (size_t)c * 64 * P + n * 64);
        };
        auto load_v = [&](int u) {
            const int slot = (tile_lo + u * UK + g * G) & (P - 1);
            const char *p = (const char *)a.c.v + (size_t)max(v_page, 0) * page_bytes + h * head_bytes + (size_t)(slot / G * D + r) * 16;
#pragma unroll
            for (int d = 0; d < DT; ++d) vf[d] = *reinterpret_cast<const uint4 *>(p + d * 256);
        };
        int u = u0 + wave;
        if (u < u1) {
            pages(u);
            load_k(u);
            load_v(u);
        }
        bool there = v_page >= 0;                                   // this lane's granule of the unit at hand
        if (u + 4 < u1) pages(u + 4);
        for (; u < u1; u += 4) {
            const bool more = u + 4 < u1;
            const int key0 = tile_lo + u * UK, key = key0 + g * G;   // key: of this lane's weights
            f32x4_t sc[RT][NK];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    sc[rt][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = NT - 1; i >= 0; --i)
#pragma unroll
                        for (int c = 0; c < KS; ++c) sc[rt][n] = mfma(operand<C>(kf[n][c / HALVES], c % HALVES), q[rt][c][i], sc[rt][n]);
                }
            if (more) load_k(u + 4);
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
                    }
#pragma unroll
                    for (int k = 0; k < PT; ++k) p[rt][hv][k] = uint4{words[k][0], words[k][1], words[k][2], words[k][3]};
                }
            }
            if (!odd_values) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int hv = 0; hv < HALVES; ++hv) {
                        const uint4 v = operand<C>(vf[d], hv);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                            for (int k = PT - 1; k >= 0; --k) acc[rt][d] = mfma(v, p[rt][hv][k], acc[rt][d]);
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
                                uint4 v = operand<C>(vf[d], hv);
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
            there = v_page >= 0;
            if (more) load_v(u + 4);
            if (u + 8 < u1) pages(u + 8);
        }
        // ---- the waves' parts
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = xor_reduce<32, 16>(l[rt], AddOp());
            if (g == 0) { m_s[wave][16 * rt + r] = m[rt]; l_s[wave][16 * rt + r] = l[rt]; }
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<float4 *>(&o_s[wave][16 * rt + r][16 * d + 4 * g]) = float4{acc[rt][d][0], acc[rt][d][1], acc[rt][d][2], acc[rt][d][3]};
        }
        __syncthreads();
        const bool alone = x0 == 0 && x1 == cost;
        const u64 item = pos - x0;
        const int wa = alone ? w : runs.of(item), wb = alone ? w : runs.of(item + cost - 1);
        constexpr int kSlot = QT * (D + 2);
        float *slot = pl.slots + (size_t)(2 * w + (w == wa)) * kSlot;
        const float v_scale = sizeof(C) == 1 ? a.c.v_scale[h] : 1.0f;
        auto finish = [&](int row, int d, float top, float sum, float (&o)[4]) {
            const int pr = t * QT + row, i = pr / group, j = pr - i * group;
            const bool empty = top == -INFINITY && sum == 0.f;
            const float by = empty ? 0.f : v_scale / sum;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = empty ? 0.f : o[k] * by;
            store_output<NT>(a, (size_t)(seq.first + i) * a.out.row + (size_t)(h * group + j) * a.out.head + d, out_wide, o);
            if (a.lse && d == 0) a.lse[(size_t)(seq.first + i) * a.n_heads + h * group + j] = empty ? -INFINITY : (top + __log2f(sum)) * kLn2;
        };
        for (int idx = tid; idx < valid * (D / 4); idx += 256) {
            const int row = idx / (D / 4), d = idx % (D / 4) * 4;
            float top = m_s[0][row], sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 1; k < 4; ++k) top = fmaxf(top, m_s[k][row]);
            const float use = top > -INFINITY ? top : 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = __builtin_amdgcn_exp2f(m_s[k][row] - use);
                const float4 x = *reinterpret_cast<const float4 *>(&o_s[k][row][d]);
                sum = __builtin_fmaf(l_s[k][row], f, sum);
                o[0] = __builtin_fmaf(x.x, f, o[0]);
                o[1] = __builtin_fmaf(x.y, f, o[1]);
                o[2] = __builtin_fmaf(x.z, f, o[2]);
                o[3] = __builtin_fmaf(x.w, f, o[3]);
            }
            if (alone) {
                finish(row, d, top, sum, o);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) agent_store(slot + row * D + d + k, o[k]);
                if (d == 0) {
                    agent_store(slot + QT * D + row, top);
                    agent_store(slot + QT * D + QT + row, sum);
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
            for (int k = wa + tid; k <= wb; k += 256)
                all_there &= __hip_atomic_load(pl.flags + 2 * k + (k == wa), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pl.number;
            if (__syncthreads_and(all_there)) {                     // (two may find so: they write the same)
                for (int idx = tid; idx < valid * (D / 4); idx += 256) {
                    const int row = idx / (D / 4), d = idx % (D / 4) * 4;
                    float top = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int k = wa; k <= wb; ++k) top = fmaxf(top, agent_load(pl.slots + (size_t)(2 * k + (k == wa)) * kSlot + QT * D + row));
                    const float use = top > -INFINITY ? top : 0.f;
                    for (int k = wa; k <= wb; ++k) {
                        const float *part = pl.slots + (size_t)(2 * k + (k == wa)) * kSlot;
                        const float f = __builtin_amdgcn_exp2f(agent_load(part + QT * D + row) - use);
                        sum = __builtin_fmaf(agent_load(part + QT * D + QT + row), f, sum);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(agent_load(part + row * D + d + e), f, o[e]);
                    }
                    finish(row, d, top, sum, o);
                }
                for (int k = wa + tid; k <= wb; k += 256)            // for the next call that carries this number (a replay)
                    __hip_atomic_store(pl.flags + 2 * k + (k == wa), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        __syncthreads();                                             // the next tile writes the waves' parts again
        pos += x1 - x0;
    }
}

// ---- launches -----------------------------------------------------------------------

constexpr int kFewGroups = 512;              // workgroups at most
static size_t slot_floats(int QT, int dim) { return (size_t)QT * (dim + 2); }

size_t paged_attention_workspace_bytes(const PagedCacheArgs &c, const PagedBatchArgs &, int) {
    return 2 * kFewGroups * sizeof(u64) + 2 * kFewGroups * slot_floats(64, c.dim) * sizeof(float);
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

hipError_t launch_paged_attention(const PagedAttentionArgs &a, hipStream_t stream) {
    PagedPlan pl;
    pl.number = call_number();
    pl.group = a.n_heads / a.c.n_kv;
    pl.flags = (u64 *)a.workspace;
    pl.slots = (float *)(pl.flags + 2 * kFewGroups);
    pl.above = 0;
    pl.upto = 0x7fffffff;
    pl.least = 192;
    const int packed = (a.b.n_rows + a.b.n_seqs - 1) / a.b.n_seqs * pl.group;
#define SPD_FEW(NT, C, D, RT)  hipLaunchKernelGGL((paged_few_kernel<NT, C, D, RT>), dim3(RT == 1 ? 512 : 256), dim3(256), 0, stream, a, pl)
#define SPD_FEW_RT(NT, C, D)                                                                                                 \
    do {                                                                                                                     \
        if (packed <= 16) SPD_FEW(NT, C, D, 1);                                                                              \
        else if (packed <= 32 || NT == 3) SPD_FEW(NT, C, D, 2);                                                              \
        else SPD_FEW(NT, C, D, (NT == 3 ? 2 : 4));                                                                           \
    } while (0)
#define SPD_FEW_D(NT, C) do { if (a.c.dim == 64) SPD_FEW_RT(NT, C, 64); else SPD_FEW_RT(NT, C, 128); } while (0)
    if (a.bf16 && a.c.e4m3) SPD_FEW_D(1, uint8_t);
    else if (a.bf16) SPD_FEW_D(1, uint16_t);
    else if (a.c.e4m3) SPD_FEW_D(3, uint8_t);
    else SPD_FEW_D(3, uint16_t);
    return hipGetLastError();
}

}  // namespace spd
