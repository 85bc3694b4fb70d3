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
template <int N>
__device__ __forceinline__ void load_n(const float *p, float (&x)[N]) {
    if constexpr (N == 8) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = p[i];
    }
}
template <int N>
__device__ __forceinline__ void load_n(const uint16_t *p, float (&x)[N]) {
    if constexpr (N == 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        x[0] = bf16_lo(a.x); x[1] = bf16_hi(a.x); x[2] = bf16_lo(a.y); x[3] = bf16_hi(a.y);
        x[4] = bf16_lo(a.z); x[5] = bf16_hi(a.z); x[6] = bf16_lo(a.w); x[7] = bf16_hi(a.w);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = bf16_bits_to_f32(p[i]);
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
    __device__ __forceinline__ void init(int part, int position, const RopeRef &r, bool inverse) {
        const int n = (IL ? r.R : r.R / 2) / E;
        turned = part < n;
        at = turned ? part * E : r.R + (part - n) * ET;
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
    // store(element, values of a run)
    template <class T, class Store>
    __device__ __forceinline__ void apply(const T *x, int R, Store store) const {
        if (!turned) {
            float v[ET];
            load_n<ET>(x + at, v);
            store(at, v);
        } else if constexpr (IL) {
            float v[E];
            load_n<E>(x + at, v);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const float a = v[2 * i], b = v[2 * i + 1];
                v[2 * i] = __builtin_fmaf(a, cs[i], -(b * sn[i]));
                v[2 * i + 1] = __builtin_fmaf(a, sn[i], b * cs[i]);
            }
            store(at, v);
        } else {
            float a[E], b[E];
            load_n<E>(x + at, a);
            load_n<E>(x + at + R / 2, b);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const float u = a[i], w = b[i];
                a[i] = __builtin_fmaf(u, cs[i], -(w * sn[i]));
                b[i] = __builtin_fmaf(u, sn[i], w * cs[i]);
            }
            store(at, a);
            store(at + R / 2, b);
        }
    }
};

constexpr int kRopeThreads = 256;

// grid: parts of all rows / 256, groups of `per` heads
template <class T, bool WIDE, bool IL>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a, int parts, int per) {
    const unsigned i = blockIdx.x * kRopeThreads + threadIdx.x;
    const unsigned row = i / (unsigned)parts;
    if (row >= (unsigned)a.n_rows) return;
    Part<WIDE, IL> part;
    part.init(i - row * parts, a.positions[row], a.rope, a.inverse);
    const int h0 = blockIdx.y * per, h1 = min(h0 + per, a.n_heads);
    const T *x = (const T *)a.x.p + row * a.x.row;
    T *out = (T *)a.out.p + row * a.out.row;
    for (int h = h0; h < h1; ++h)
        part.apply(x + h * a.x.head, a.rope.R, [&](int at, const auto &v) { store_n(out + h * a.out.head + at, v); });
}

// ---- append -----------------------------------------------------------------------

// the sequence that `row` belongs to; n_seqs: none
__device__ __forceinline__ int seq_of(const PagedBatchArgs &b, int row) {
    if (!b.row_start) return row / b.each;
    int lo = 0, hi = b.n_seqs;                               // the last sequence that starts at or before the row
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (b.row_start[mid] <= row) lo = mid; else hi = mid;
    }
    int first, last;
    paged_rows(b, lo, first, last);
    return row >= first && row < last ? lo : b.n_seqs;
}

struct E4m3 { uint8_t x; };
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

// grid: parts of all rows / 256, groups of `per` heads: of the queries, then of the keys, then of the values
template <class T, class C, bool WIDE, bool IL>
__global__ __launch_bounds__(kRopeThreads) void paged_append_kernel(PagedAppendArgs a, int parts, int per, int q_groups, int k_groups) {
    constexpr int G = 16 / sizeof(C);
    const unsigned i = blockIdx.x * kRopeThreads + threadIdx.x;
    const unsigned row = i / (unsigned)parts;
    if (row >= (unsigned)a.b.n_rows) return;
    const int seq = seq_of(a.b, row);
    if (seq >= a.b.n_seqs) return;
    int first, last;
    paged_rows(a.b, seq, first, last);
    const int p = paged_len(a.b, seq) + ((int)row - first), P = 1 << a.c.page_bits, slot = p & (P - 1);
    const int group = blockIdx.y, kind = group < q_groups ? 0 : (group < q_groups + k_groups ? 1 : 2);
    const int h0 = (group - (kind == 0 ? 0 : (kind == 1 ? q_groups : q_groups + k_groups))) * per, h1 = min(h0 + per, kind == 0 ? a.n_heads : a.c.n_kv);
    Part<WIDE, IL> part;
    RopeRef rope = a.rope;
    if (kind == 2) rope.R = 0;
    if ((int)(i - row * parts) >= Part<WIDE, IL>::count(rope.R, a.c.dim, true)) return;      // turned heads have fewer parts
    part.init(i - row * parts, a.positions ? a.positions[row] : p, rope, false);
    if (kind == 0) {
        for (int h = h0; h < h1; ++h)
            part.apply((const T *)a.q.p + row * a.q.row + h * a.q.head, rope.R,
                       [&](int at, const auto &v) { store_n((T *)a.q_out.p + row * a.q_out.row + h * a.q_out.head + at, v); });
        return;
    }
    const int page = paged_page(a.b, a.c, seq, p >> a.c.page_bits);
    if (page < 0) return;
    const HeadsArgs &src = kind == 1 ? a.k : a.v;
    const float *scales = kind == 1 ? a.c.k_scale : a.c.v_scale;
    for (int h = h0; h < h1; ++h) {
        C *dst = (C *)(kind == 1 ? a.c.k : a.c.v) + ((size_t)page * a.c.n_kv + h) * a.c.dim * P;
        const float scale = scales ? scales[h] : 1.0f;
        part.apply((const T *)src.p + row * src.row + h * src.head, rope.R, [&](int at, const auto &v) {
            if (kind == 1) {
                put_held(dst + ((size_t)(at / G) * P + slot) * G + at % G, v, scale);
            } else {
                constexpr int N = sizeof(v) / sizeof(float);
                C *to = dst + ((size_t)(slot / G) * a.c.dim + at) * G + slot % G;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float one[1] = {v[e]};
                    put_held(to + e * G, one, scale);
                }
            }
        });
    }
}

// ---- launches ----------------------------------------------------------------------

hipError_t launch_rope_table(const RopeTableArgs &a, void *table, hipStream_t stream) {
    hipLaunchKernelGGL(rope_table_kernel, dim3(1), dim3(128), 0, stream, a, (char *)table);
    return hipGetLastError();
}

static bool wide_heads(const HeadsArgs &h, int size) { return (uintptr_t)h.p % 16 == 0 && h.row * size % 16 == 0 && h.head * size % 16 == 0; }
static bool wide_rope(const RopeRef &r, int dim) { return dim % 8 == 0 && r.R % (r.interleaved ? 8 : 16) == 0; }
// heads a thread takes: more share the sines and cosines, fewer fill the CUs
static int heads_per_thread(size_t threads, int heads) {
    int per = 8;
    while (per > 1 && threads * ((heads + per - 1) / per) < 256 * 1024) per /= 2;
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
#define SPD_APPEND(T, C, W, I)                                                                                               \
    do {                                                                                                                     \
        const int parts = std::max(Part<W, I>::count(a.rope.R, a.c.dim, true), Part<W, I>::count(0, a.c.dim, true));         \
        const size_t threads = (size_t)parts * a.b.n_rows;                                                                   \
        const int per = heads_per_thread(threads, a.n_heads + 2 * a.c.n_kv);                                                 \
        const int qg = a.q.p ? (a.n_heads + per - 1) / per : 0, kg = (a.c.n_kv + per - 1) / per;                             \
        hipLaunchKernelGGL((paged_append_kernel<T, C, W, I>), dim3((threads + kRopeThreads - 1) / kRopeThreads, qg + 2 * kg), dim3(kRopeThreads), 0, stream, a, parts, per, qg, kg); \
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
