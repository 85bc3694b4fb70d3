// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits (or probabilities).
//
//   z = l / T,   lp(x) = z_x - log sum exp z,   entropy = -sum p lp
//   rank of a token = entries before it in descending order, equal ones by index
//
// Order is an integer: the bits of a float32 as an ordered 32-bit key over the complement of the index, so that no two
// entries are equal and every choice has one answer.
#include "launch.h"

namespace spd {

constexpr int kLpThreads = 1024;

__device__ __forceinline__ uint32_t ordered_bits(float v) {    // ascending as v does; both zeros alike
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

template <class T, class Op>
__device__ T block_reduce(T v, T *tmp, Op op) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = op(v, (T)__shfl_xor(v, m, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    v = tmp[0];
    for (int i = 1; i < kLpThreads / 64; ++i) v = op(v, tmp[i]);
    return v;
}

// One workgroup per row, any vocabulary size: the row is walked in memory.
__global__ __launch_bounds__(kLpThreads) void logprobs_kernel(LogprobArgs a) {
    const size_t r = blockIdx.x;
    const float *row = a.rows + r * a.row_stride;
    const int V = a.vocab;
    __shared__ unsigned long long tmp64[kLpThreads / 64];
    __shared__ float tmp[kLpThreads / 64];
    const int token = a.tokens ? a.tokens[r] : -1;
    const bool known = token >= 0 && token < V;
    const float mine = known ? row[token] : 0.f;
    float mx = -INFINITY;
    bool bad = false;
    unsigned long long before = 0;
    for (int x = threadIdx.x; x < V; x += kLpThreads) {
        const float v = row[x];
        bad |= !(v < INFINITY) || (a.probs && !(v >= 0.f));
        mx = fmaxf(mx, v);
        before += v > mine || (v == mine && x < token);
    }
    mx = block_reduce(mx, tmp, [](float x, float y) { return fmaxf(x, y); });
    bad = block_reduce((unsigned long long)bad, tmp64, [](unsigned long long x, unsigned long long y) { return x | y; }) != 0;
    before = block_reduce(before, tmp64, [](unsigned long long x, unsigned long long y) { return x + y; });
    const float lowest = a.probs ? 0.f : -INFINITY;            // entries at it have no mass
    const bool empty = !(mx > lowest);
    float sum = 0.f, dot = 0.f;                                // of e and e * (z - max), or of p log p
    if (!bad && !empty)
        for (int x = threadIdx.x; x < V; x += kLpThreads) {
            const float v = row[x];
            if (!(v > lowest)) continue;
            if (a.probs) dot += v * logf(v);
            else {
                const float d = (v - mx) * a.inv_temp, e = expf(d);
                sum += e;
                dot += e > 0.f ? e * d : 0.f;
            }
        }
    sum = block_reduce(sum, tmp, [](float x, float y) { return x + y; });
    dot = block_reduce(dot, tmp, [](float x, float y) { return x + y; });
    const float log_sum = a.probs ? 0.f : logf(sum);
    auto lp = [&](float v) { return a.probs ? logf(v) : (v - mx) * a.inv_temp - log_sum; };
    const float nan = __uint_as_float(0x7fc00000u);
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[r] = bad ? nan : (known && mine > lowest ? lp(mine) : -INFINITY);
        if (a.rank) a.rank[r] = bad ? -1 : (known ? (int)before : V);
        if (a.entropy) a.entropy[r] = bad ? nan : (empty ? 0.f : (a.probs ? -dot : log_sum - dot / sum));
    }
    unsigned long long bound = ~0ull;                          // keys below it are left
    for (int i = 0; i < a.n_top; ++i) {
        unsigned long long best = 0;
        if (!bad)
            for (int x = threadIdx.x; x < V; x += kLpThreads) {
                const float v = row[x];
                const unsigned long long key = (unsigned long long)ordered_bits(v) << 32 | (uint32_t)~x;
                if (v > lowest && key < bound && key > best) best = key;
            }
        best = block_reduce(best, tmp64, [](unsigned long long x, unsigned long long y) { return x > y ? x : y; });
        bound = best;
        if (threadIdx.x == 0) {
            a.top_tokens[r * a.n_top + i] = best ? (int)~(uint32_t)best : -1;
            a.top_logprobs[r * a.n_top + i] = bad ? nan : (best ? lp(from_ordered((uint32_t)(best >> 32))) : -INFINITY);
        }
    }
}

size_t logprobs_workspace_bytes(int n_rows, int vocab, int n_top) { (void)n_rows; (void)vocab; (void)n_top; return 0; }

hipError_t launch_logprobs(const LogprobArgs &a, hipStream_t stream) {
    hipLaunchKernelGGL(logprobs_kernel, dim3(a.n_rows), dim3(kLpThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace spd
