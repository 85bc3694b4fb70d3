// Attention of the new rows of sequences over their pages.
#include "paged.h"

namespace spd {

template <class C> __device__ __forceinline__ float held(C x);
template <> __device__ __forceinline__ float held<uint16_t>(uint16_t x) { return bf16_bits_to_f32(x); }
template <> __device__ __forceinline__ float held<uint8_t>(uint8_t x) { return __builtin_amdgcn_cvt_f32_fp8(x, 0); }

// One wave per (row, head): a lane scores a key, then owns D / 64 elements of the output.
template <class T, class C, int D>
__global__ __launch_bounds__(64) void paged_attention_simple_kernel(PagedAttentionArgs a) {
    constexpr int G = 16 / sizeof(C), N = D / 64;
    const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, kvh = h / (a.n_heads / a.c.n_kv);
    int seq = 0, first = 0, last = 0;
    for (seq = 0; seq < a.b.n_seqs; ++seq) {
        paged_rows(a.b, seq, first, last);
        if (row >= first && row < last) break;
    }
    if (seq == a.b.n_seqs) return;
    const int len = paged_len(a.b, seq), i = row - first, P = 1 << a.c.page_bits, p = len + i;
    __shared__ float q[D], w[64];
    for (int d = lane; d < D; d += 64) {
        const size_t at = row * a.q.row + h * a.q.head + d;
        q[d] = a.bf16 ? bf16_bits_to_f32(((const uint16_t *)a.q.p)[at]) : ((const float *)a.q.p)[at];
    }
    const float ks = a.c.k_scale ? a.c.k_scale[kvh] : 1.f, vs = a.c.v_scale ? a.c.v_scale[kvh] : 1.f;
    const uint64_t bits = a.seen ? a.seen[row] : 0;
    const int end = min(a.seen ? len + min(last - first, 64) : p + 1, a.b.capacity);
    const int begin = a.window ? max(0, p - a.window + 1) : 0;
    float m = -INFINITY, l = 0.f, acc[N] = {};
    __syncthreads();
    for (int k0 = begin; k0 < end; k0 += 64) {
        const int key = k0 + lane;
        bool sees = key < end && (!a.seen || key < len || (bits >> (key - len) & 1));
        const int page = sees ? paged_page(a.b, a.c, seq, key >> a.c.page_bits) : -1;
        sees = sees && page >= 0;
        float s = -INFINITY;
        if (sees) {
            const C *kp = (const C *)a.c.k + ((size_t)page * a.c.n_kv + kvh) * D * P + (key & (P - 1)) * G;
            s = 0.f;
            for (int d = 0; d < D; ++d) s = __builtin_fmaf(q[d], held<C>(kp[(size_t)(d / G) * P * G + d % G]), s);
            s *= ks * a.scale;
        }
        const float mx = fmaxf(m, wave_max(s)), use = mx > -INFINITY ? mx : 0.f;
        const float shrink = m > -INFINITY ? expf(m - use) : 0.f, e = s == -INFINITY ? 0.f : expf(s - use);
        l = l * shrink + wave_sum(e);
        m = mx;
        w[lane] = e;
        __syncthreads();
        for (int n = 0; n < N; ++n) acc[n] *= shrink;
        for (int j = 0; j < 64; ++j) {
            const int kj = k0 + j, pj = __shfl(page, j);
            if (pj < 0) continue;
            for (int n = 0; n < N; ++n) {
                const int d = lane + 64 * n, slot = kj & (P - 1);
                const C *vp = (const C *)a.c.v + ((size_t)pj * a.c.n_kv + kvh) * D * P;
                acc[n] = __builtin_fmaf(w[j], held<C>(vp[((size_t)(slot / G) * D + d) * G + slot % G]), acc[n]);
            }
        }
        __syncthreads();
    }
    const bool empty = m == -INFINITY && l == 0.f;
    for (int n = 0; n < N; ++n) {
        const float y = empty ? 0.f : acc[n] / l * vs;
        const size_t at = row * a.out.row + h * a.out.head + lane + 64 * n;
        if (a.bf16) ((uint16_t *)a.out.p)[at] = f32_to_bf16_bits(y);
        else ((float *)a.out.p)[at] = y;
    }
    if (a.lse && lane == 0) a.lse[(size_t)row * a.n_heads + h] = empty ? -INFINITY : m + logf(l);
}

size_t paged_attention_workspace_bytes(const PagedCacheArgs &, const PagedBatchArgs &, int) { return 256; }

hipError_t launch_paged_attention(const PagedAttentionArgs &a, hipStream_t stream) {
    const dim3 grid(a.b.n_rows, a.n_heads);
    if (a.c.dim == 64 && a.c.e4m3) hipLaunchKernelGGL((paged_attention_simple_kernel<float, uint8_t, 64>), grid, dim3(64), 0, stream, a);
    else if (a.c.dim == 64) hipLaunchKernelGGL((paged_attention_simple_kernel<float, uint16_t, 64>), grid, dim3(64), 0, stream, a);
    else if (a.c.e4m3) hipLaunchKernelGGL((paged_attention_simple_kernel<float, uint8_t, 128>), grid, dim3(64), 0, stream, a);
    else hipLaunchKernelGGL((paged_attention_simple_kernel<float, uint16_t, 128>), grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace spd
