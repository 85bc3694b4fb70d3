// Rotary positions, and appending keys (turned on the way) and values to a paged cache.
//
//   (a, b) -> m (a cos t - b sin t, a sin t + b cos t),  t = position * f_i
//
// A frequency is a 64-bit fraction of a turn: position * frequency modulo 2^64 is the angle's place within its turn, exact, however far the
// position.  What is left is within an eighth of a turn of a quarter, where sine and cosine are their Taylor sums.
#include <algorithm>

#include "paged.h"

namespace spd {

__global__ void rope_table_kernel(RopeTableArgs a, char *table) {
    if (threadIdx.x == 0) *reinterpret_cast<float *>(table) = a.magnitude;
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) reinterpret_cast<uint64_t *>(table + kRopeHeader)[i] = a.turn[i];
}

// sine and cosine of position * turn (2^-64 turns); the remainder x is within pi / 4, where the first terms left out are x^11 / 11! < 1.8e-9
// and x^12 / 12! < 1.2e-10
__device__ __forceinline__ void turn_of(int position, uint64_t turn, float &sn, float &cs) {
    const uint32_t at = (uint32_t)(((uint64_t)(int64_t)position * turn) >> 32);      // place within the turn, 2^-32 turns
    const uint32_t quarter = (at + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(at - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
    const float y = x * x;
    const float s = __builtin_fmaf(x * y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 2.7557319224e-6f, -1.9841269841e-4f), 8.3333333333e-3f), -1.6666666667e-1f), x);
    const float c = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -2.7557319224e-7f, 2.4801587302e-5f), -1.3888888889e-3f), 4.1666666667e-2f), -0.5f), 1.0f);
    const float a = (quarter & 1) ? c : s, b = (quarter & 1) ? s : c;
    sn = (quarter & 2) ? -a : a;
    cs = ((quarter + 1) & 2) ? -b : b;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_bits_to_f32(x); }
__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t *p, float x) { *p = f32_to_bf16_bits(x); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) float f32x2_t;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
// N neighbouring elements; 8 of them by loads and stores of 16 bytes
template <int N, class T>
__device__ __forceinline__ void load_n(const T *p, T (&x)[N]) {
    if constexpr (N == 8) {
        uint4 q[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = reinterpret_cast<const uint4 *>(p)[i];
        __builtin_memcpy(x, q, sizeof(x));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = p[i];
    }
}
template <int N>
__device__ __forceinline__ void store_n(float *p, const float (&x)[N]) {
    if constexpr (N == 8) {
        reinterpret_cast<float4 *>(p)[0] = float4{x[0], x[1], x[2], x[3]};
        reinterpret_cast<float4 *>(p)[1] = float4{x[4], x[5], x[6], x[7]};
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = x[i];
    }
}
template <int N>
__device__ __forceinline__ void store_n(uint16_t *p, const float (&x)[N]) {
    if constexpr (N == 8) {
        *reinterpret_cast<uint4 *>(p) = uint4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = f32_to_bf16_bits(x[i]);
    }
}

// What a thread does with its part of a head: a pair of runs of elements (half layout: i .. and i + R / 2 ..), one run (interleaved), or a run behind
// the turned part.  WIDE: runs of 8, else single pairs and elements.  Sines and cosines are made once for all heads that the thread takes.
template <bool WIDE, bool IL>
struct Part {
    static constexpr int E = WIDE ? 8 : (IL ? 2 : 1);        // elements a run
    static constexpr int ET = WIDE ? 8 : 1;                  // ... behind the turned part
    static constexpr int NP = IL ? E / 2 : E;                // pairs
    float sn[NP], cs[NP];
    int at;                                                  // first element
    bool turned;
    // parts of a head; without the rest where it stays in place
    static __host__ __device__ int count(int R, int dim, bool rest) { return (IL ? R : R / 2) / E + (rest ? (dim - R) / ET : 0); }
    __device__ __forceinline__ void init(int part, const RopeRef &r) {
        const int n = (IL ? r.R : r.R / 2) / E;
        turned = part < n;
        at = turned ? part * E : r.R + (part - n) * ET;
    }
    __device__ __forceinline__ void angles(int position, const RopeRef &r, bool inverse) {
        if (!turned) return;
        const float m = *reinterpret_cast<const float *>(r.table);
        const uint64_t *turn = reinterpret_cast<const uint64_t *>((const char *)r.table + kRopeHeader) + (IL ? at / 2 : at);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            turn_of(position, turn[i], sn[i], cs[i]);
            sn[i] *= inverse ? -m : m;
            cs[i] *= m;
        }
    }
    // What the thread reads of a head, as it lies there: loads may be under way while something else is found out
    template <class T>
    struct Raw { T a[E], b[IL ? 1 : E], rest[ET]; };
    template <class T>
    __device__ __forceinline__ void load(const T *x, int R, Raw<T> &raw) const {
        if (!turned) {
            load_n<ET>(x + at, raw.rest);
        } else {
            load_n<E>(x + at, raw.a);
            if constexpr (!IL) load_n<E>(x + at + R / 2, raw.b);
        }
    }
    // store(element, values of a run)
    template <class T, class Store>
    __device__ __forceinline__ void apply(const Raw<T> &raw, int R, Store store) const {
        if (!turned) {
            float v[ET];
#pragma unroll
            for (int i = 0; i < ET; ++i) v[i] = to_f32(raw.rest[i]);
            store(at, v);
        } else if constexpr (IL) {
            float v[E];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const float a = to_f32(raw.a[2 * i]), b = to_f32(raw.a[2 * i + 1]);
                v[2 * i] = __builtin_fmaf(a, cs[i], -(b * sn[i]));
                v[2 * i + 1] = __builtin_fmaf(a, sn[i], b * cs[i]);
            }
            store(at, v);
        } else {
            float v[E], w[E];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const float a = to_f32(raw.a[i]), b = to_f32(raw.b[i]);
                v[i] = __builtin_fmaf(a, cs[i], -(b * sn[i]));
                w[i] = __builtin_fmaf(a, sn[i], b * cs[i]);
            }
            store(at, v);
            store(at + R / 2, w);
        }
    }
};

constexpr int kRopeThreads = 256;

// grid: parts of all rows / 256, groups of `per` heads.  Bound by memory: 8192 rows of 32 heads of 128 in bf16 29.1 us, 4.6 TB/s read and written (a plain copy
// reaches 4.9); 3001 rows of 20 heads of 96 in float32, 40 of them turned in neighbouring pairs, 9.8 us.  A single row is a launch, 3.1 us.  The sines and
// cosines of a pair (some 30 instructions) are made once for all heads that the thread takes, and a head's loads are under way while the one before is turned.
template <class T, bool WIDE, bool IL>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a, int parts, int per) {
    const unsigned i = blockIdx.x * kRopeThreads + threadIdx.x;
    const unsigned row = i / (unsigned)parts;
    if (row >= (unsigned)a.n_rows) return;
    Part<WIDE, IL> part;
    part.init(i - row * parts, a.rope);
    const int h0 = blockIdx.y * per, h1 = min(h0 + per, a.n_heads);
    const T *x = (const T *)a.x.p + row * a.x.row;
    T *out = (T *)a.out.p + row * a.out.row;
    typename Part<WIDE, IL>::template Raw<T> raw;
    part.load(x + h0 * a.x.head, a.rope.R, raw);
    part.angles(a.positions[row], a.rope, a.inverse);
    for (int h = h0; h < h1; ++h) {
        const auto now = raw;
        if (h + 1 < h1) part.load(x + (h + 1) * a.x.head, a.rope.R, raw);
        part.apply(now, a.rope.R, [&](int at, const auto &v) { store_n(out + h * a.out.head + at, v); });
    }
}

// ---- append -----------------------------------------------------------------------

// The batch's rows and lengths: in LDS where they fit
struct BatchRows {
    const int32_t *starts, *lens;
    // the sequence that `row` belongs to, its first row and the one behind its last; n_seqs: none
    __device__ __forceinline__ int find(const PagedBatchArgs &b, int row, int &first, int &last) const {
        if (!b.row_start) {
            const int seq = row / b.each;
            first = seq * b.each;
            last = first + b.each;
            return seq;
        }
        int lo = 0, hi = b.n_seqs;                           // the last sequence that starts at or before the row
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (starts[mid] <= row) lo = mid; else hi = mid;
        }
        first = min(max(starts[lo], 0), b.n_rows);
        last = min(max(starts[lo + 1], first), b.n_rows);
        return row >= first && row < last ? lo : b.n_seqs;
    }
    __device__ __forceinline__ int len(const PagedBatchArgs &b, int seq) const { return min(max(lens[seq], 0), b.capacity); }
};

__device__ __forceinline__ float to_held(float x, float scale) {       // x / scale within e4m3's range, NaN kept
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(x / scale, -448.0f), 448.0f);
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// a run of N elements into a granule of keys
template <int N>
__device__ __forceinline__ void put_held(uint16_t *p, const float (&x)[N], float) { store_n(p, x); }
template <int N>
__device__ __forceinline__ void put_held(uint8_t *p, const float (&x)[N], float scale) {
    float y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = to_held(x[i], scale);
    if constexpr (N == 8) *reinterpret_cast<uint2 *>(p) = uint2{pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7])};
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = (uint8_t)pack_e4m3(y[i], 0.f, 0.f, 0.f);
    }
}

constexpr int kStartsInLds = 1024;

// Values: a wave takes a head of `block` rows, a lane D / 64 dims of it.  Where a granule's slots are all of this call, the lane has the granule together
// and writes its 16 bytes (rows of 64 lanes side by side); a part of one is written element by element, so that the slots beside it stay as they are.
// (A thread a row and 8 dims, 8 stores of 2 bytes each: 7100 rows of 32 + 8 + 8 heads of 128 75 us, now 41.)
template <class T, class C, int N>
__device__ __forceinline__ void append_values(const PagedAppendArgs &a, const BatchRows &rows, int unit, int block) {
    constexpr int G = 16 / sizeof(C);
    const int lane = threadIdx.x & 63, h = unit % a.c.n_kv, row0 = unit / a.c.n_kv * block, P = 1 << a.c.page_bits;
    // a lane per row: which rows begin a granule (or their sequence)
    const int row = row0 + lane;
    int seq = a.b.n_seqs, first = 0, last = 0, p = 0;
    if (lane < block && row < a.b.n_rows) seq = rows.find(a.b, row, first, last);
    if (seq < a.b.n_seqs) p = rows.len(a.b, seq) + (row - first);
    unsigned long long begins = __ballot(seq < a.b.n_seqs && (row == first || p % G == 0));
    const float scale = a.c.v_scale ? a.c.v_scale[h] : 1.0f;
    while (begins) {
        const int l = __builtin_ctzll(begins);
        begins &= begins - 1;
        const int s = __builtin_amdgcn_readlane(seq, l), pos = __builtin_amdgcn_readlane(p, l), end = __builtin_amdgcn_readlane(last, l);
        const int r0 = row0 + l, slot = pos & (P - 1), n = min(G - slot % G, end - r0);
        const T *src = (const T *)a.v.p + h * a.v.head + lane * N;
        T raw[G][N];                                             // on their way together with the page
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) raw[i][e] = src[(size_t)(r0 + min(i, n - 1)) * a.v.row + e];
        const int page = paged_page(a.b, a.c, s, pos >> a.c.page_bits);
        if (page < 0) continue;                                  // a granule lies in one page
        float x[G][N];
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) x[i][e] = to_f32(raw[i][e]);
        C *dst = (C *)a.c.v + (((size_t)page * a.c.n_kv + h) * (P / G) + slot / G) * a.c.dim * G + lane * N * G;
        if (n == G) {
#pragma unroll
            for (int e = 0; e < N; ++e)
#pragma unroll
                for (int i = 0; i < G; i += 8) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = x[i + k][e];
                    put_held(dst + e * G + i, y, scale);
                }
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (i < n) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float one[1] = {x[i][e]};
                        put_held(dst + e * G + slot % G + i, one, scale);
                    }
                }
        }
    }
}

// workgroups of values; rows a wave of them; parts of a row's head, heads a thread, groups of heads (of q; all), workgroups a group
struct AppendGrid { int values_first, value_groups, block, parts, per, q_groups, groups, across; };

// Bound by memory where rows are many: 7100 rows of 32 + 8 + 8 heads of 128 in bf16 41.6 us, 4.2 TB/s; by the way from the batch's rows to a place and its
// stores where they are few: 5 rows of 3 x 32 heads 4.4 us, 2400 rows of 16 + 4 + 4 heads of 64 in e4m3 9.4.  What a row is stays in LDS (searched there: a step in
// memory is a third of a microsecond), and the loads of a head begin before its place is known.
// grid: the values, four waves a workgroup, and groups of `per` heads, of the queries and of the keys, by the parts of all rows / 256
template <class T, class C, bool WIDE, bool IL>
__global__ __launch_bounds__(kRopeThreads) void paged_append_kernel(PagedAppendArgs a, AppendGrid g) {
    constexpr int G = 16 / sizeof(C);
    __shared__ int32_t starts[kStartsInLds + 1], lens[kStartsInLds];
    BatchRows rows{a.b.row_start, a.b.lens};
    const bool in_lds = a.b.row_start && a.b.n_seqs <= kStartsInLds;
    if (in_lds)
        for (int i = threadIdx.x; i <= a.b.n_seqs; i += kRopeThreads) {
            starts[i] = a.b.row_start[i];
            if (i < a.b.n_seqs) lens[i] = a.b.lens[i];
        }
    const int turned = g.groups * g.across, in_values = (int)blockIdx.x - (g.values_first ? 0 : turned);
    if (in_values >= 0 && in_values < g.value_groups) {
        const int unit = in_values * 4 + (threadIdx.x >> 6);
        if (in_lds) { __syncthreads(); rows = BatchRows{starts, lens}; }
        if (unit / a.c.n_kv * g.block >= a.b.n_rows) return;
        if (a.c.dim == 64) append_values<T, C, 1>(a, rows, unit, g.block);
        else append_values<T, C, 2>(a, rows, unit, g.block);
        return;
    }
    const int block = (int)blockIdx.x - (g.values_first ? g.value_groups : 0), group = block / g.across;
    const unsigned i = (block - group * g.across) * kRopeThreads + threadIdx.x, row = i / (unsigned)g.parts;
    const bool keys = group >= g.q_groups, mine = row < (unsigned)a.b.n_rows;
    const int h0 = (keys ? group - g.q_groups : group) * g.per, h1 = min(h0 + g.per, keys ? a.c.n_kv : a.n_heads);
    const HeadsArgs &src = keys ? a.k : a.q;
    const T *x = (const T *)src.p + row * src.row;
    Part<WIDE, IL> part;
    part.init(i - row * g.parts, a.rope);
    typename Part<WIDE, IL>::template Raw<T> raw;
    if (mine) part.load(x + h0 * src.head, a.rope.R, raw);
    if (in_lds) { __syncthreads(); rows = BatchRows{starts, lens}; }
    if (!mine) return;
    int first, last;
    const int seq = rows.find(a.b, row, first, last);
    if (seq >= a.b.n_seqs) return;
    const int p = rows.len(a.b, seq) + ((int)row - first), page = keys ? paged_page(a.b, a.c, seq, p >> a.c.page_bits) : 0;
    if (page < 0) return;
    part.angles(a.positions ? a.positions[row] : p, a.rope, false);
    const int P = 1 << a.c.page_bits, slot = p & (P - 1);
    for (int h = h0; h < h1; ++h) {
        const auto now = raw;
        if (h + 1 < h1) part.load(x + (h + 1) * src.head, a.rope.R, raw);
        if (keys) {
            C *dst = (C *)a.c.k + ((size_t)page * a.c.n_kv + h) * a.c.dim * P;
            const float scale = a.c.k_scale ? a.c.k_scale[h] : 1.0f;
            part.apply(now, a.rope.R, [&](int at, const auto &v) { put_held(dst + ((size_t)(at / G) * P + slot) * G + at % G, v, scale); });
        } else {
            part.apply(now, a.rope.R, [&](int at, const auto &v) { store_n((T *)a.q_out.p + row * a.q_out.row + h * a.q_out.head + at, v); });
        }
    }
}

// ---- launches ----------------------------------------------------------------------

hipError_t launch_rope_table(const RopeTableArgs &a, void *table, hipStream_t stream) {
    hipLaunchKernelGGL(rope_table_kernel, dim3(1), dim3(128), 0, stream, a, (char *)table);
    return hipGetLastError();
}

static bool wide_heads(const HeadsArgs &h, int size) { return (uintptr_t)h.p % 16 == 0 && h.row * size % 16 == 0 && h.head * size % 16 == 0; }
static bool wide_rope(const RopeRef &r, int dim) { return dim % 8 == 0 && r.R % (r.interleaved ? 8 : 16) == 0; }
// heads a thread takes: more share the sines and cosines, fewer fill the CUs (2400 rows of 16 + 4 + 4 heads of 64: 10.0 us with 256 Ki threads asked for, 9.5 with 64 Ki)
static int heads_per_thread(size_t threads, int heads) {
    int per = 8;
    while (per > 1 && threads * ((heads + per - 1) / per) < 64 * 1024) per /= 2;
    return per;
}

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream) {
    const int size = a.bf16 ? 2 : 4;
    const bool wide = wide_rope(a.rope, a.dim) && wide_heads(a.x, size) && wide_heads(a.out, size);
    const bool rest = a.x.p != a.out.p;
#define SPD_ROPE(T, W, I)                                                                                                    \
    do {                                                                                                                     \
        const int parts = Part<W, I>::count(a.rope.R, a.dim, rest);                                                          \
        const size_t threads = (size_t)parts * a.n_rows;                                                                     \
        const int per = heads_per_thread(threads, a.n_heads);                                                                \
        hipLaunchKernelGGL((rope_kernel<T, W, I>), dim3((threads + kRopeThreads - 1) / kRopeThreads, (a.n_heads + per - 1) / per), dim3(kRopeThreads), 0, stream, a, parts, per); \
    } while (0)
#define SPD_ROPE_I(T, W) do { if (a.rope.interleaved) SPD_ROPE(T, W, true); else SPD_ROPE(T, W, false); } while (0)
    if (a.bf16 && wide) SPD_ROPE_I(uint16_t, true);
    else if (a.bf16) SPD_ROPE_I(uint16_t, false);
    else if (wide) SPD_ROPE_I(float, true);
    else SPD_ROPE_I(float, false);
    return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t stream) {
    const int size = a.bf16 ? 2 : 4;
    const bool wide = (!a.rope.table || wide_rope(a.rope, a.c.dim)) && wide_heads(a.k, size) && wide_heads(a.v, size) && (!a.q.p || (wide_heads(a.q, size) && wide_heads(a.q_out, size)));
    // Rows of values a wave: a granule's where that leaves enough waves, else one (the wave of a granule's first row takes all of it)
    const int granule = a.c.e4m3 ? 16 : 8;
    AppendGrid g;
    g.block = (size_t)a.b.n_rows * a.c.n_kv >= (size_t)granule * 256 ? granule : 1;
    g.value_groups = (int)(((size_t)((a.b.n_rows + g.block - 1) / g.block) * a.c.n_kv + 3) / 4);
    // Few of them start first, as a wave of values waits longest; many would hold the others up: 2400 rows of 16 + 4 + 4 heads of 64 in e4m3, 155 workgroups,
    // 9.7 us first and 11.5 last; 7100 rows of 32 + 8 + 8 heads of 128, 1775 workgroups, 46 and 41.  The border is no sharp one: 2100 rows of the latter, 524 workgroups,
    // 15.3 and 14.0, 1400 rows, 350, 12.0 and 11.3, and in e4m3, 174, 16.0 and 13.5; 700 rows, 86, 11.4 and 11.8.
    g.values_first = g.value_groups <= 512;
#define SPD_APPEND(T, C, W, I)                                                                                               \
    do {                                                                                                                     \
        g.parts = Part<W, I>::count(a.rope.R, a.c.dim, true);                                                                \
        const size_t threads = (size_t)g.parts * a.b.n_rows;                                                                 \
        g.per = heads_per_thread(threads, a.n_heads + a.c.n_kv);                                                             \
        g.q_groups = a.q.p ? (a.n_heads + g.per - 1) / g.per : 0;                                                            \
        g.groups = g.q_groups + (a.c.n_kv + g.per - 1) / g.per;                                                              \
        g.across = (int)((threads + kRopeThreads - 1) / kRopeThreads);                                                       \
        hipLaunchKernelGGL((paged_append_kernel<T, C, W, I>), dim3((unsigned)(g.groups * g.across) + (unsigned)g.value_groups), dim3(kRopeThreads), 0, stream, a, g); \
    } while (0)
#define SPD_APPEND_I(T, C, W) do { if (a.rope.interleaved) SPD_APPEND(T, C, W, true); else SPD_APPEND(T, C, W, false); } while (0)
#define SPD_APPEND_W(T, C) do { if (wide) SPD_APPEND_I(T, C, true); else SPD_APPEND_I(T, C, false); } while (0)
    if (a.bf16 && a.c.e4m3) SPD_APPEND_W(uint16_t, uint8_t);
    else if (a.bf16) SPD_APPEND_W(uint16_t, uint16_t);
    else if (a.c.e4m3) SPD_APPEND_W(float, uint8_t);
    else SPD_APPEND_W(float, uint16_t);
    return hipGetLastError();
}

}  // namespace spd
