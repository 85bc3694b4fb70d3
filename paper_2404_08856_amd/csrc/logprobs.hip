// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits (or probabilities).
//
//   z = l / T,   lp(x) = z_x - log sum exp z,   entropy = -sum p lp
//   rank of a token = entries before it in descending order, equal ones by index
//
// Order is an integer: the bits of a float32 as an ordered 32-bit key over the complement of the index, so that no two
// entries are equal and every choice has one answer.
#include <algorithm>

#include "launch.h"
#include "row_quads.h"

namespace spd {

__device__ __forceinline__ uint32_t ordered_bits(float v) {    // ascending as v does; both zeros alike
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ unsigned long long order_key(float v, int x) { return (unsigned long long)ordered_bits(v) << 32 | (uint32_t)~x; }

struct MaximumOp { __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_elementwise_maximum(a, b); } };   // NaN stays
struct MinimumOp { __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_elementwise_minimum(a, b); } };

// What a row, or a slice of it, comes to.  Of logits: sum of e = 2^((l - mx) / (T ln 2)), and of e times that exponent; of
// probabilities: dot = sum p log2 p.
struct LpPart { float mx, mn, sum, dot; unsigned before; };

constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;

// The row's answers from its whole part; `mine`: the token's entry
struct LpFinish {
    const LogprobArgs &a;
    LpPart p;
    bool bad, empty;
    float log_sum, lowest;
    __device__ __forceinline__ LpFinish(const LogprobArgs &a_, const LpPart &p_) : a(a_), p(p_) {
        lowest = a.probs ? 0.f : -INFINITY;
        bad = !(p.mx < INFINITY) || (a.probs && !(p.mn >= 0.f));
        empty = !(p.mx > lowest);
        log_sum = a.probs ? 0.f : logf(p.sum);
    }
    // (halves: the difference of two float32 may be beyond float32 where its T-th is not)
    __device__ __forceinline__ float lp(float v) const { return a.probs ? logf(v) : 2.0f * __builtin_fmaf(0.5f * v - 0.5f * p.mx, a.inv_temp, -0.5f * log_sum); }
    __device__ __forceinline__ void write(size_t r, int token, float mine) const {
        const float nan = __uint_as_float(0x7fc00000u);
        const bool known = token >= 0 && token < a.vocab;
        if (a.logprob) a.logprob[r] = bad ? nan : (known && mine > lowest ? lp(mine) : -INFINITY);
        if (a.rank) a.rank[r] = bad ? -1 : (known ? (int)p.before : a.vocab);
        if (a.entropy) a.entropy[r] = bad ? nan : (empty ? 0.f : (a.probs ? -kLn2 * p.dot : log_sum - kLn2 * (p.dot / p.sum)));
    }
    // alternative i; key 0: there is none
    __device__ __forceinline__ void alternative(size_t r, int i, unsigned long long key) const {
        a.top_tokens[r * a.n_top + i] = !bad && key ? (int)~(uint32_t)key : -1;
        a.top_logprobs[r * a.n_top + i] = bad ? __uint_as_float(0x7fc00000u) : (key ? lp(from_ordered((uint32_t)(key >> 32))) : -INFINITY);
    }
};

__device__ __forceinline__ float exponent2(float v, float mx, float scale2) {      // at least -200, where 2^x is 0 as it is at -infinity (and 0 * x is 0)
    return fmaxf((v - mx) * scale2, -200.f);
}

// Partial results of a slice in the workspace
struct LpRecord { LpPart p; unsigned pad[3]; };

// The wave's 64 values in descending order over the lanes (bitonic: 21 exchanges)
template <int SIZE, int N>
__device__ __forceinline__ float sort_step(float v, int lane) {
    const float o = lane_xor<N>(v);
    v = ((lane & N) != 0) == ((lane & SIZE) != 0) ? fmaxf(v, o) : fminf(v, o);
    if constexpr (N > 1) v = sort_step<SIZE, N / 2>(v, lane);
    return v;
}
template <int SIZE = 2>
__device__ __forceinline__ float sort_descending(float v, int lane) {
    v = sort_step<SIZE, SIZE / 2>(v, lane);
    if constexpr (SIZE < 64) v = sort_descending<SIZE * 2>(v, lane);
    return v;
}

// One workgroup per row, or per slice of one of at most THREADS * NV quads; the entries stay in registers.
//
// Alternatives: the n-th largest of 64 bucket maxima (a bucket is what the lanes of one number hold) is a bound that at least n
// entries reach, and for entries in no particular order few more than n do (32 of 64 buckets: about 44).  Those are listed in
// LDS, and each finds its place by counting the keys above it.  Where more than kListed reach it (equal entries,
// rows whose first ones all fall on a few lanes) the maximum is taken n times instead, from memory (2048 rows of 32000 equal entries, 5 alternatives: 340 us).
//
// Many rows are bound by memory: 2048 x 32000 50 us (262 MB: 5.2 TB/s; on other cards up to 59), 320 x 32003 14.6.  One row of 32000 is 7.3 us: its entries' way from
// memory, two exchanges over the workgroup, the list.  Rows over several workgroups would add another's end and start to that (see the merge).
constexpr int kListed = 256;
template <int THREADS, int NV, bool ALIGNED, bool PROBS>
__global__ __launch_bounds__(THREADS, 8) void logprobs_kernel(LogprobArgs a, int slices, int slice_quads) {
    constexpr int WAVES = THREADS / 64;
    const int r = blockIdx.x / slices, slice = blockIdx.x - r * slices;
    const float *row = a.rows + (size_t)r * a.row_stride;
    const int V = a.vocab, lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q0 = slice * slice_quads, n4 = (V + 3) >> 2, q1 = min(n4, q0 + slice_quads);
    __shared__ float s_max[WAVES][64], s_min[WAVES], s_sum[WAVES], s_dot[WAVES], s_bound;
    __shared__ unsigned s_before[WAVES], s_count;
    __shared__ unsigned long long s_key[kListed];
    constexpr float lowest = PROBS ? 0.f : -INFINITY;

    float4 v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int q = q0 + i * THREADS + (int)threadIdx.x;
        v[i] = load_quad<ALIGNED>(row, q < q1 ? q : n4, V, lowest);
    }
    const int token = a.tokens ? a.tokens[r] : -1;
    const bool known = token >= 0 && token < V;
    const float mine = known ? row[token] : 0.f;
    if (threadIdx.x == 0) s_count = 0;

    float top = -INFINITY, low = INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        top = MaximumOp()(top, MaximumOp()(MaximumOp()(v[i].x, v[i].y), MaximumOp()(v[i].z, v[i].w)));
        if (PROBS) low = MinimumOp()(low, MinimumOp()(MinimumOp()(v[i].x, v[i].y), MinimumOp()(v[i].z, v[i].w)));
    }
    s_max[w][lane] = top;
    if (PROBS) {
        low = xor_reduce<32, 1>(low, MinimumOp());
        if (lane == 0) s_min[w] = low;
    }
    __syncthreads();
    LpPart p;
    float bucket = s_max[0][lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) bucket = MaximumOp()(bucket, s_max[i][lane]);
    p.mx = xor_reduce<32, 1>(bucket, MaximumOp());
    p.mn = 0.f;
    if (PROBS) {
        p.mn = s_min[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) p.mn = MinimumOp()(p.mn, s_min[i]);
    }
    if (w == 0 && a.n_top > 0) {                              // the n-th largest bucket (one of NaN: any bound will do)
        const float sorted = sort_descending(bucket, lane);
        if (lane == a.n_top - 1) s_bound = sorted;
    }
    float sum = 0.f, dot = 0.f;
    if (p.mx > lowest) {
        const float scale2 = a.inv_temp * kLog2e;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float e4[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (PROBS) dot += e4[j] >= 0x1p-126f ? e4[j] * __log2f(e4[j]) : 0.f;      // (of less the instruction takes no logarithm; they would add less than 2^-119)
                else {
                    const float d = exponent2(e4[j], p.mx, scale2), e = __builtin_amdgcn_exp2f(d);
                    sum += e;
                    dot = __builtin_fmaf(e, d, dot);
                }
            }
        }
    }
    unsigned before = 0;
    if (a.rank && known) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int first = 4 * (q0 + i * THREADS + 64 * w);      // of the wave's 256 entries
            const float e4[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            if (first + 255 < token && first + 256 <= 4 * q1) {
#pragma unroll
                for (int j = 0; j < 4; ++j) before += e4[j] >= mine;
            } else if (first > token) {
#pragma unroll
                for (int j = 0; j < 4; ++j) before += e4[j] > mine;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) before += e4[j] > mine || (e4[j] == mine && first + 4 * lane + j < min(token, 4 * q1));
            }
        }
    }
    sum = wave_sum(sum);
    dot = wave_sum(dot);
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) before += (unsigned)__shfl_xor((int)before, m, 64);
    if (lane == 0) { s_sum[w] = sum; s_dot[w] = dot; s_before[w] = before; }
    __syncthreads();
    p.sum = p.dot = 0.f;
    p.before = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { p.sum += s_sum[i]; p.dot += s_dot[i]; p.before += s_before[i]; }
    const LpFinish f(a, p);
    if (threadIdx.x == 0) {
        if (slices == 1) f.write(r, token, mine);
        else reinterpret_cast<LpRecord *>(a.workspace)[blockIdx.x].p = p;
    }
    if (a.n_top == 0) return;
    unsigned long long *keys = reinterpret_cast<unsigned long long *>(reinterpret_cast<LpRecord *>(a.workspace) + (size_t)a.n_rows * slices) + (size_t)blockIdx.x * a.n_top;
    auto place = [&](int i, unsigned long long key) __attribute__((always_inline)) {
        if (slices == 1) f.alternative(r, i, key);
        else keys[i] = key;
    };
    const float bound = s_bound;
    if (f.bad) {                                              // (a slice that is not: the merge sees the others')
        if ((int)threadIdx.x < a.n_top) place(threadIdx.x, 0);
        return;
    }
    if (top >= bound && top > lowest) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float e4[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            if (!(fmaxf(fmaxf(e4[0], e4[1]), fmaxf(e4[2], e4[3])) >= bound)) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e4[j] >= bound && e4[j] > lowest) {
                    const unsigned at = atomicAdd(&s_count, 1u);
                    if (at < kListed) s_key[at] = order_key(e4[j], 4 * (q0 + i * THREADS + (int)threadIdx.x) + j);
                }
        }
    }
    __syncthreads();
    const int count = (int)s_count;
    if (count <= kListed) {
        if ((int)threadIdx.x < count) {
            const unsigned long long key = s_key[threadIdx.x];
            int above = 0;
            for (int i = 0; i < count; ++i) above += s_key[i] > key;
            if (above < a.n_top) place(above, key);
        }
        if ((int)threadIdx.x < a.n_top && (int)threadIdx.x >= count) place(threadIdx.x, 0);
        return;
    }
    unsigned long long last = ~0ull;                          // keys below it are left
    for (int n = 0; n < a.n_top; ++n) {
        unsigned long long best = 0;
        for (int x = 4 * q0 + (int)threadIdx.x; x < min(V, 4 * q1); x += THREADS) {
            const float e = row[x];
            const unsigned long long key = order_key(e, x);
            if (e > lowest && key < last && key > best) best = key;
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) {
            const unsigned long long o = __shfl_xor(best, m, 64);
            best = o > best ? o : best;
        }
        __syncthreads();                                      // the list, or the round before, has been read
        if (lane == 0) s_key[w] = best;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) best = s_key[i] > best ? s_key[i] : best;
        last = best;
        if (threadIdx.x == 0) place(n, best);
    }
}

// Rows in slices: one workgroup per row joins what the slices left.  Both launches: one row of 131072 10.4 us, 64 15.6 (34 MB), 4 rows of 2^20 16.
constexpr int kMergeThreads = 256;
__global__ __launch_bounds__(kMergeThreads) void logprobs_merge_kernel(LogprobArgs a, int slices) {
    constexpr int WAVES = kMergeThreads / 64;
    const size_t r = blockIdx.x;
    const LpRecord *rec = reinterpret_cast<const LpRecord *>(a.workspace) + r * slices;
    const unsigned long long *keys = reinterpret_cast<const unsigned long long *>(reinterpret_cast<const LpRecord *>(a.workspace) + (size_t)a.n_rows * slices) + r * slices * a.n_top;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    __shared__ LpPart s_part[WAVES];
    __shared__ unsigned long long s_key[kListed];
    const int token = a.tokens ? a.tokens[r] : -1;
    const float mine = token >= 0 && token < a.vocab ? a.rows[r * a.row_stride + token] : 0.f;
    LpPart p = {-INFINITY, INFINITY, 0.f, 0.f, 0};
    for (int i = threadIdx.x; i < slices; i += kMergeThreads) {
        p.mx = MaximumOp()(p.mx, rec[i].p.mx);
        p.mn = MinimumOp()(p.mn, rec[i].p.mn);
        p.before += rec[i].p.before;
    }
    p.mx = xor_reduce<32, 1>(p.mx, MaximumOp());
    p.mn = xor_reduce<32, 1>(p.mn, MinimumOp());
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) p.before += (unsigned)__shfl_xor((int)p.before, m, 64);
    if (lane == 0) s_part[w] = p;
    __syncthreads();
    p = s_part[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) {
        p.mx = MaximumOp()(p.mx, s_part[i].mx);
        p.mn = MinimumOp()(p.mn, s_part[i].mn);
        p.before += s_part[i].before;
    }
    float sum = 0.f, dot = 0.f;
    for (int i = threadIdx.x; i < slices; i += kMergeThreads) {
        const LpPart s = rec[i].p;
        if (a.probs) dot += s.dot;
        else if (s.mx > -INFINITY) {
            const float d = exponent2(s.mx, p.mx, a.inv_temp * kLog2e), e = __builtin_amdgcn_exp2f(d);
            sum += e * s.sum;
            dot += e * __builtin_fmaf(s.sum, d, s.dot);
        }
    }
    sum = wave_sum(sum);
    dot = wave_sum(dot);
    __syncthreads();
    if (lane == 0) { s_part[w].sum = sum; s_part[w].dot = dot; }
    __syncthreads();
    p.sum = p.dot = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { p.sum += s_part[i].sum; p.dot += s_part[i].dot; }
    const LpFinish f(a, p);
    if (threadIdx.x == 0) f.write(r, token, mine);
    if (a.n_top == 0) return;
    const size_t n = (size_t)slices * a.n_top;
    if (f.bad) {
        if ((int)threadIdx.x < a.n_top) f.alternative(r, threadIdx.x, 0);
        return;
    }
    if (n <= kListed) {                                       // the places of keys among all; keys of nothing (0) come last, in order
        if (threadIdx.x < n) s_key[threadIdx.x] = keys[threadIdx.x];
        __syncthreads();
        if (threadIdx.x >= n) return;
        const unsigned long long key = s_key[threadIdx.x];
        int above = 0;
        for (int i = 0; i < (int)n; ++i) above += s_key[i] > key || (s_key[i] == key && i < (int)threadIdx.x);
        if (above < a.n_top) f.alternative(r, above, key);
        return;
    }
    unsigned long long last = ~0ull;
    for (int t = 0; t < a.n_top; ++t) {
        unsigned long long best = 0;
        for (size_t i = threadIdx.x; i < n; i += kMergeThreads)
            if (keys[i] < last && keys[i] > best) best = keys[i];
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) {
            const unsigned long long o = __shfl_xor(best, m, 64);
            best = o > best ? o : best;
        }
        __syncthreads();
        if (lane == 0) s_key[w] = best;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) best = s_key[i] > best ? s_key[i] : best;
        last = best;
        if (threadIdx.x == 0) f.alternative(r, t, best);
    }
}

// both factors that the kernels take of it are numbers: an infinite one makes NaN of the largest entry's 0
bool logprob_temperature_ok(float temperature) {
    const float inv = 1.0f / temperature;
    return temperature > 0.f && inv > 0.f && inv * kLog2e < INFINITY;
}

constexpr int kSliceEntries = 32768;      // what a workgroup of 1024 holds in registers
int logprob_slices(int vocab) { return (int)(((long)vocab + kSliceEntries - 1) / kSliceEntries); }

size_t logprobs_workspace_bytes(int n_rows, int vocab, int n_top) {
    const size_t slices = logprob_slices(vocab);
    return slices == 1 ? 0 : n_rows * slices * (sizeof(LpRecord) + n_top * sizeof(unsigned long long));
}

template <int THREADS, int NV>
static void launch_rows(const LogprobArgs &a, int slices, int slice_quads, hipStream_t stream) {
    const bool aligned = ((uintptr_t)a.rows & 15) == 0 && (a.row_stride & 3) == 0 && (a.vocab & 3) == 0;
    const dim3 grid((unsigned)((size_t)a.n_rows * slices)), block(THREADS);
    if (aligned && a.probs) hipLaunchKernelGGL((logprobs_kernel<THREADS, NV, true, true>), grid, block, 0, stream, a, slices, slice_quads);
    else if (aligned) hipLaunchKernelGGL((logprobs_kernel<THREADS, NV, true, false>), grid, block, 0, stream, a, slices, slice_quads);
    else if (a.probs) hipLaunchKernelGGL((logprobs_kernel<THREADS, NV, false, true>), grid, block, 0, stream, a, slices, slice_quads);
    else hipLaunchKernelGGL((logprobs_kernel<THREADS, NV, false, false>), grid, block, 0, stream, a, slices, slice_quads);
}

// Threads per row: the fewest that hold it in at most 8 quads each, and not fewer than are worth a row's own latency.  Alternatives
// (us for 1, 320, 2048 rows): 1000 entries with 4 quads 4.4, 5.4, 8.8 instead of 3.9, 4.5, 7.0; 4096 in 1024 threads 4.3, 6.2, 18.6 instead of
// 4.4, 5.5, 10.8; 8192 in 256 x 8 5.4, 6.8, 15.9 and in 1024 4.6, 6.8, 21.7 instead of 4.6, 6.3, 16.1; 16384 in 1024 5.4, 10.0, 32.6 instead of 5.4, 9.8, 27.6.
hipError_t launch_logprobs(const LogprobArgs &a, hipStream_t stream) {
    const int slices = logprob_slices(a.vocab), n4 = (a.vocab - 1) / 4 + 1;
    const int per = (n4 + slices - 1) / slices;
    if (per <= 256) launch_rows<256, 1>(a, slices, per, stream);
    else if (per <= 1024) launch_rows<256, 4>(a, slices, per, stream);
    else if (per <= 2048) launch_rows<512, 4>(a, slices, per, stream);
    else if (per <= 4096) launch_rows<512, 8>(a, slices, per, stream);
    else launch_rows<1024, 8>(a, slices, per, stream);
    if (slices > 1) hipLaunchKernelGGL(logprobs_merge_kernel, dim3(a.n_rows), dim3(kMergeThreads), 0, stream, a, slices);
    return hipGetLastError();
}

}  // namespace spd
