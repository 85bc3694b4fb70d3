// Weights in 4 bits: the quantiser, its inverse, the re-tiling and the product  Y[rows, N] = X[rows, K] W[N, K]^T  for up
// to 64 rows, with the epilogues of the decoder's projections.
//
//   W[n][k] = scale[n][k / G] * q[n][k],   q in -8 .. 7,   scale bfloat16,   G = 32, 64 or 128
//
// The product is made of integers.  The values of an activation row in a block of 128 columns (many rows: a chunk of blocks) share the exponent E of their
// largest magnitude: x = v * 2^(E - 30) with a 31-bit integer v, and v is four signed base-256 digits.  v is off by at most one, half where |x| is small: one
// is at most 2^-29 of the largest magnitude; or by 2^-23 of itself where that is more.  On a row of normal values the digits add 6e-9 to a product's
// error of 2.2e-7; a value 3000 times the others' makes their error (as seen in outputs where its own weight is 0) 2.5e-7 in a block of 128, 5.7e-7 in a
// chunk of 512, one of 30000 times 2e-6 and 4e-6 (K = 4096).  Four rows x four digits are the 16
// rows of v_mfma_i32_16x16x64_i8; a nibble in the upper half of a byte is 16 q as an 8-bit integer, so the weights need
// one mask (and every other one a shift) per 4 of them and no zero point.  The sums of a group are exact in 32 bits (at most
// 128 * 128 * 128 = 2^21 a digit), those of two neighbouring digits together as well (2^30).  A lane ends with the four digits' sums of one
// activation row and one output: two shift-and-adds, two conversions and a fused multiply-add make their float32 value (rounded three times), a product
// with the scale and another fused multiply-add with 2^(E - 34) bring it into the output's float32 sum.
// A row with a value that is not finite gives NaN; a block whose largest magnitude is below 2^-90 keeps less than 31 bits.
// (One product in bfloat16 takes the matrix core as long as one here, and float32's accuracy takes three terms of each activation there,
// four digits here; but there each weight has to be made from its nibble, here a mask does.)
#include <algorithm>

#include "launch.h"

namespace spd {

typedef __attribute__((ext_vector_type(4))) int i32x4_t;

constexpr int kQ4Block = 128;             // columns of a block: 16 bytes per lane of a 16-row tile
constexpr int kQ4Rows = 4;                // activation rows of a row group

// ---------------------------------------------------------------------------------
// quantiser and its inverse, row-major
// ---------------------------------------------------------------------------------
struct __attribute__((packed, aligned(4))) FloatQuad { float v[4]; };
struct __attribute__((packed, aligned(2))) HalfOct { uint32_t v[4]; };
struct __attribute__((packed, aligned(1))) ByteQuad { uint32_t v; };

// values k0 .. k0 + 7 of a row of K, zeros behind its end.  ONCE: nobody reads them again
template <bool ONCE = false>
__device__ __forceinline__ void load8(const float *row, size_t k0, int K, float (&v)[8]) {
    typedef __attribute__((ext_vector_type(4), aligned(4))) float quad_t;
    if (k0 + 8 <= (size_t)K) {
        const quad_t *p = reinterpret_cast<const quad_t *>(row + k0), *r = reinterpret_cast<const quad_t *>(row + k0 + 4);
        const quad_t a = ONCE ? __builtin_nontemporal_load(p) : *p, b = ONCE ? __builtin_nontemporal_load(r) : *r;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k0 + e < (size_t)K ? row[k0 + e] : 0.f;
    }
}
template <bool ONCE = false>
__device__ __forceinline__ void load8(const uint16_t *row, size_t k0, int K, float (&v)[8]) {
    typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t quad_t;
    if (k0 + 8 <= (size_t)K) {
        const quad_t *p = reinterpret_cast<const quad_t *>(row + k0);
        const quad_t a = ONCE ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = bf16_lo(a[e]); v[2 * e + 1] = bf16_hi(a[e]); }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k0 + e < (size_t)K ? bf16_bits_to_f32(row[k0 + e]) : 0.f;
    }
}

// A wave per 512 columns of a row, 8 per lane; a group is 4, 8 or 16 neighbouring lanes.  Bound by memory: 4096 x 4096 bf16 12.7 us (42 MB, 3.3 TB/s).  With its inverse
// behind it 26.5 (118 MB) and 11003 x 4099 float32 83.6 (408 MB: 4.9 TB/s; on another card 74.7); loads that are not non-temporal 28.4 and 86.1, a quotient per
// weight 1.3 more and 0.6, two and four units per wave 29.2 / 87.4 and 33.4 / 90.2, non-temporal stores in the inverse 33.1 / 106.7.
template <class T, int G>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const T *__restrict__ W, size_t ldw, int N, int K, uint8_t *__restrict__ q, uint16_t *__restrict__ scales) {
    const int per_row = (K + 511) / 512, lane = threadIdx.x & 63;
    const unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);         // (at most 2^26: a division in 64 bits is 100 instructions)
    if (unit >= (unsigned)N * per_row) return;
    const unsigned r = unit / (unsigned)per_row;
    const size_t n = r, k0 = (size_t)(unit - r * per_row) * 512 + lane * 8;
    float v[8];
    load8<true>(W + n * ldw, k0, K, v);
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = __builtin_elementwise_maximum(m, fabsf(v[e]));        // NaN stays
    m = __builtin_elementwise_maximum(m, lane_xor<1>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<2>(m));
    if (G >= 64) m = __builtin_elementwise_maximum(m, lane_xor<4>(m));
    if (G >= 128) m = __builtin_elementwise_maximum(m, lane_xor<8>(m));
    const bool finite = m < INFINITY;
    const uint16_t s16 = finite ? f32_to_bf16_bits(m * (1.0f / 7.0f)) : (uint16_t)0x7fc0;
    const float s = bf16_bits_to_f32(s16);
    // w / s by a product with 1 / s, off by at most 2^-19 (|w / s| < 8): only next to a tie does the quotient itself decide
    const bool some = finite && s != 0.f;
    const float inv = 1.0f / s;
    uint32_t bytes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e] * inv;
        float near = rintf(x);
        if (!(fabsf(x - near) < 0.49999f)) near = rintf(v[e] / s);
        const int i = some ? (int)fminf(fmaxf(near, -8.f), 7.f) : 0;
        bytes |= (uint32_t)(i & 15) << (4 * e);                // even columns in the low halves
    }
    if (k0 >= (size_t)K) return;
    if (k0 % G == 0) scales[n * ((K + G - 1) / G) + k0 / G] = s16;
    const size_t row_bytes = ((size_t)K + 1) / 2;
    uint8_t *dst = q + n * row_bytes + k0 / 2;
    if (k0 + 8 <= (size_t)K) reinterpret_cast<ByteQuad *>(dst)->v = bytes;
    else
        for (size_t e = 0; k0 / 2 + e < row_bytes; ++e) dst[e] = (uint8_t)(bytes >> (8 * e));
}

// 8 columns per thread.  Bound by memory: 4096 x 4096 to bf16 10.6 us (42 MB, 4.0 TB/s), to float32 15.5 (76 MB, 4.9 TB/s)
template <class T, int G>
__global__ __launch_bounds__(256) void q4_dequantize_kernel(const uint8_t *__restrict__ q, const uint16_t *__restrict__ scales, int N, int K, T *__restrict__ W, size_t ldw) {
    const int per_row = (K + 511) / 512, lane = threadIdx.x & 63;
    const unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);         // (at most 2^26: a division in 64 bits is 100 instructions)
    if (unit >= (unsigned)N * per_row) return;
    const unsigned r = unit / (unsigned)per_row;
    const size_t n = r, k0 = (size_t)(unit - r * per_row) * 512 + lane * 8;
    if (k0 >= (size_t)K) return;
    const size_t row_bytes = ((size_t)K + 1) / 2;
    const uint8_t *src = q + n * row_bytes + k0 / 2;
    uint32_t bytes = 0;
    if (k0 + 8 <= (size_t)K) bytes = reinterpret_cast<const ByteQuad *>(src)->v;
    else
        for (size_t e = 0; k0 / 2 + e < row_bytes; ++e) bytes |= (uint32_t)src[e] << (8 * e);
    const float s = bf16_bits_to_f32(scales[n * ((K + G - 1) / G) + k0 / G]);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)((int)(bytes << (28 - 4 * e)) >> 28) * s;
    T *dst = W + n * ldw + k0;
    if (k0 + 8 <= (size_t)K) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<FloatQuad *>(dst) = FloatQuad{{v[0], v[1], v[2], v[3]}};
            *reinterpret_cast<FloatQuad *>(dst + 4) = FloatQuad{{v[4], v[5], v[6], v[7]}};
        } else {
            HalfOct o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o.v[e] = f32_to_bf16_bits(v[2 * e]) | (uint32_t)f32_to_bf16_bits(v[2 * e + 1]) << 16;
            *reinterpret_cast<HalfOct *>(dst) = o;
        }
    } else {
        for (size_t e = 0; k0 + e < (size_t)K; ++e) {
            if constexpr (sizeof(T) == 4) dst[e] = v[e];
            else dst[e] = f32_to_bf16_bits(v[e]);
        }
    }
}

bool q4_group_ok(int G) { return G == 32 || G == 64 || G == 128; }

template <class F>
static hipError_t with_group(int G, F f) {
    switch (G) {
        case 32: f(std::integral_constant<int, 32>()); break;
        case 64: f(std::integral_constant<int, 64>()); break;
        case 128: f(std::integral_constant<int, 128>()); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

static unsigned unit_grid(int N, int K) { return (unsigned)(((size_t)N * ((K + 511) / 512) + 3) / 4); }

hipError_t launch_q4_quantize(const void *W, bool bf16, size_t ldw, int N, int K, int G, void *q, void *scales, hipStream_t stream) {
    return with_group(G, [&](auto g) {
        if (bf16) hipLaunchKernelGGL((q4_quantize_kernel<uint16_t, g()>), dim3(unit_grid(N, K)), dim3(256), 0, stream, (const uint16_t *)W, ldw, N, K, (uint8_t *)q, (uint16_t *)scales);
        else hipLaunchKernelGGL((q4_quantize_kernel<float, g()>), dim3(unit_grid(N, K)), dim3(256), 0, stream, (const float *)W, ldw, N, K, (uint8_t *)q, (uint16_t *)scales);
    });
}

hipError_t launch_q4_dequantize(const void *q, const void *scales, int N, int K, int G, void *W, bool bf16, size_t ldw, hipStream_t stream) {
    return with_group(G, [&](auto g) {
        if (bf16) hipLaunchKernelGGL((q4_dequantize_kernel<uint16_t, g()>), dim3(unit_grid(N, K)), dim3(256), 0, stream, (const uint8_t *)q, (const uint16_t *)scales, N, K, (uint16_t *)W, ldw);
        else hipLaunchKernelGGL((q4_dequantize_kernel<float, g()>), dim3(unit_grid(N, K)), dim3(256), 0, stream, (const uint8_t *)q, (const uint16_t *)scales, N, K, (float *)W, ldw);
    });
}

// ---------------------------------------------------------------------------------
// re-tiling
// ---------------------------------------------------------------------------------
// Tiles of 16 rows, blocks of 128 columns: block (t, b) at index t * KB + b is 1 KiB, lane l = r + 16 g holds row 16 t + r in its
// 16 bytes: word j < 4 has columns 128 b + 32 j + 8 g + e (e < 4) in the upper halves of its bytes and + 4 + e in the lower
// ones.  Two masks make of words 2 s, 2 s + 1 the operand of matrix-core step s (64 columns, in an order that the activations follow).
// Behind the blocks the scales, [t][b][16 rows][128 / G].
// Rows and columns beyond the matrix are zero.  A wave writes a block; a lane reads 4 times 4 bytes of its row (4096 x 4096: 8.3 us, 17 MB; once a model).
size_t q4_scales_offset(int N, int K) { return ((size_t)((N + 15) / 16) * ((K + kQ4Block - 1) / kQ4Block) * 1024 + 255) / 256 * 256; }
size_t q4_packed_bytes(int N, int K, int G) {
    return (q4_scales_offset(N, K) + (size_t)((N + 15) / 16) * ((K + kQ4Block - 1) / kQ4Block) * (4096 / G) + 255) / 256 * 256;
}

struct Q4PackArgs {
    const uint8_t *q[3];
    const uint16_t *s[3];
    int mode, N, K, KB, G;
    uint4 *blocks;
    uint16_t *scales;
};
// source matrix and row of packed row p; false beyond the matrix
__device__ __forceinline__ bool source_row(const Q4PackArgs &a, int p, int &which, int &row) {
    which = 0; row = p;
    if (a.mode == PACK_CONCAT3) {
        const int third = a.N / 3;
        which = min(p / third, 2);
        row = p - which * third;
    } else if (a.mode == PACK_GATE_UP) {
        which = (p & 15) >= 8;
        row = (p >> 4) * 8 + (p & 7);
    }
    return p < a.N;
}
__global__ __launch_bounds__(256) void q4_pack_kernel(Q4PackArgs a) {
    const size_t id = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6), tiles = (size_t)(a.N + 15) / 16;
    if (id >= tiles * a.KB) return;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int t = (int)(id / a.KB), b = (int)(id - (size_t)t * a.KB);
    int which, row;
    const size_t row_bytes = ((size_t)a.K + 1) / 2;
    uint32_t w[4] = {0, 0, 0, 0};
    if (source_row(a, 16 * t + r, which, row)) {
        const uint8_t *src = a.q[which] + (size_t)row * row_bytes;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k0 = kQ4Block * b + 32 * j + 8 * g;
            uint32_t v = 0;                                    // 8 columns as they lie
            if (k0 + 8 <= a.K) v = reinterpret_cast<const ByteQuad *>(src + k0 / 2)->v;
            else
                for (int k = k0; k < a.K; ++k) v |= (uint32_t)(src[k >> 1] >> (4 * (k & 1)) & 15) << (4 * (k - k0));
            auto spread = [](uint32_t x) { x = (x | x << 8) & 0x00ff00ffu; return (x | x << 4) & 0x0f0f0f0fu; };     // nibble i of 4 to byte i
            w[j] = spread(v & 0xffffu) << 4 | spread(v >> 16);
        }
    }
    a.blocks[id * 64 + lane] = uint4{w[0], w[1], w[2], w[3]};
    const int per = kQ4Block / a.G, groups = (a.K + a.G - 1) / a.G;      // scales of the block: 16 rows x per
    for (int i = lane; i < 16 * per; i += 64) {                          // [row][per]
        const int group = b * per + i % per;
        uint16_t v = 0;
        if (group < groups && source_row(a, 16 * t + i / per, which, row)) v = a.s[which][(size_t)row * groups + group];
        a.scales[id * (16 * per) + i] = v;
    }
}

hipError_t launch_q4_pack(const void *const (&q)[3], const void *const (&scales)[3], int mode, int N, int K, int G, void *packed, hipStream_t stream) {
    if (!q4_group_ok(G)) return hipErrorInvalidValue;
    Q4PackArgs a;
    for (int i = 0; i < 3; ++i) { a.q[i] = (const uint8_t *)q[i]; a.s[i] = (const uint16_t *)scales[i]; }
    a.mode = mode; a.N = N; a.K = K; a.KB = (K + kQ4Block - 1) / kQ4Block; a.G = G;
    a.blocks = (uint4 *)packed;
    a.scales = (uint16_t *)((char *)packed + q4_scales_offset(N, K));
    const size_t blocks = (size_t)((N + 15) / 16) * a.KB;
    hipLaunchKernelGGL(q4_pack_kernel, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// For prompts: a wave per block of 128 columns writes its four blocks of 32 in bf16 and their rows' factors.  Bound by memory: 22016 x 4096 40.4 us (237 MB, 5.9 TB/s),
// 8 % of the time of a 640-row prompt in all.  (The same in the prompt kernel would be made anew for every 64 rows.)
template <int G>
__global__ __launch_bounds__(256) void q4_unpack_kernel(const uint4 *__restrict__ W, const uint16_t *__restrict__ S, int KB, int KS, int tile0, size_t blocks,
                                                        uint4 *__restrict__ out, float *__restrict__ wscale) {
    const size_t id = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= blocks) return;
    const int lane = threadIdx.x & 63, t = (int)(id / KB), b = (int)(id - (size_t)t * KB);
    const size_t src = (size_t)tile0 * KB + id;
    const uint4 w = W[src * 64 + lane];
    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (4 * b + j >= KS) break;
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {                          // columns 2 e, 2 e + 1 of the lane's 8
            auto value = [&](int k) { return (float)((int)(words[j] << (24 - 8 * (k & 3) + (k < 4 ? 0 : 4))) >> 28); };
            p[e] = f32_to_bf16_bits(value(2 * e)) | (uint32_t)f32_to_bf16_bits(value(2 * e + 1)) << 16;
        }
        out[((size_t)t * KS + 4 * b + j) * 64 + lane] = uint4{p[0], p[1], p[2], p[3]};
    }
    const int j = lane >> 4, row = lane & 15;
    if (4 * b + j < KS) wscale[((size_t)t * KS + 4 * b + j) * 16 + row] = bf16_bits_to_f32(S[(src * 16 + row) * (kQ4Block / G) + 32 * j / G]);
}

hipError_t launch_q4_unpack(const void *packed, int N, int K, int G, int tile0, int n_tiles, void *blocks, float *wscale, hipStream_t stream) {
    const int KB = (K + kQ4Block - 1) / kQ4Block;
    const size_t n = (size_t)n_tiles * KB;
    return with_group(G, [&](auto g) {
        hipLaunchKernelGGL(q4_unpack_kernel<g()>, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, stream, (const uint4 *)packed,
                           (const uint16_t *)((const char *)packed + q4_scales_offset(N, K)), KB, (K + 31) / 32, tile0, n, (uint4 *)blocks, wscale);
    });
}

// ---------------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------------
struct Q4Kernel {
    const uint4 *W;
    const uint16_t *S;
    int N, K, KB, tiles;
    const void *X;
    int x_kind;               // Q4_X_F32, Q4_X_BF16 (row-major, ldx elements apart) or Q4_X_PACKED (three bf16 terms, KS blocks a row group)
    size_t ldx;
    int KS, row0, rows;       // rows of the call; this launch starts at row0
    float *Y;
    size_t ldy;
    const float *ssq_in;      // the rest as in GemmArgs
    int ssq_in_parts;
    float inv_d, eps;
    const float *gain_next;
    float *Xnext;
    float *ssq_out;
    float *Xout;
    int K_out, epilogue;
};

// Values k0 .. k0 + 7 (k0 % 8 == 0) of an activation row, zeros beyond the matrix
template <int KIND>
__device__ __forceinline__ void load_x8(const Q4Kernel &a, int row, int k0, float (&v)[8]) {
    if (row >= a.rows || k0 >= a.K) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
    } else if constexpr (KIND == Q4_X_F32) {
        load8((const float *)a.X + (size_t)row * a.ldx, k0, a.K, v);
    } else if constexpr (KIND == Q4_X_BF16) {
        load8((const uint16_t *)a.X + (size_t)row * a.ldx, k0, a.K, v);
    } else {                                                   // the sum of the terms is the float32 value they were made of
        const uint16_t *X = (const uint16_t *)a.X;
        uint4 t[kTerms];
#pragma unroll
        for (int i = 0; i < kTerms; ++i) t[i] = *reinterpret_cast<const uint4 *>(X + xpack_index(row, k0, a.KS, i));
        const uint32_t *p0 = &t[0].x, *p1 = &t[1].x, *p2 = &t[2].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = bf16_lo(p0[e]) + (bf16_lo(p1[e]) + bf16_lo(p2[e]));
            v[2 * e + 1] = bf16_hi(p0[e]) + (bf16_hi(p1[e]) + bf16_hi(p2[e]));
        }
    }
}
// f(KIND) for the call's kind of activations: the branch stands around all loads of a unit, not around each
template <class F>
__device__ __forceinline__ void with_kind(const Q4Kernel &a, F f) {
    if (a.x_kind == Q4_X_F32) f(std::integral_constant<int, Q4_X_F32>());
    else if (a.x_kind == Q4_X_BF16) f(std::integral_constant<int, Q4_X_BF16>());
    else f(std::integral_constant<int, Q4_X_PACKED>());
}

__device__ __forceinline__ uint32_t byte_perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

// Digits of a block of 128 columns for a row group.  Lane l = (4 c + t) + 16 g brings columns 32 t + 8 g .. + 7 of row c
// and leaves with digit t (t = 3: the leading one) of columns 32 j + 8 g .. + 7, j < 4, of the row: B[2 j], B[2 j + 1].
// exponent: of the largest magnitude among what the lane's row has there (biased, at least 36, 255: not finite).
__device__ __forceinline__ int shared_exponent(float m) {      // m: the lane's largest magnitude, or NaN
    m = __builtin_elementwise_maximum(m, lane_xor<1>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<2>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<16>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<32>(m));
    return max((int)(__float_as_uint(m) >> 23 & 255u), 36);
}
__device__ __forceinline__ int block_exponent(const float (&v)[8]) {
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = __builtin_elementwise_maximum(m, fabsf(v[e]));        // NaN stays
    return shared_exponent(m);
}
// What a sum of 16 q * v is worth, 2^(E - 34), is small where the activations are, and times a small scale below any float32 while the result is
// not.  So the scales meet the sums first: up to 2^44 a block, 2^56 a chunk, times 2^-32 of the scale, which the factor bears instead: scales up to 2^100 stay in
// range, and those down to 2^-100 keep their 8 bits.
constexpr int kQ4ScaleShift = 32;
constexpr float kQ4ScaleDown = 0x1p-32f;
__device__ __forceinline__ float digit_factor(int exponent) {
    return exponent == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((unsigned)(exponent - 33 + kQ4ScaleShift) << 23);
}
__device__ __forceinline__ void block_digits(const float (&v)[8], int exponent, uint32_t (&B)[8]) {
    const float up = __uint_as_float((unsigned)(283 - exponent) << 23);       // 2^(30 - E): |v| stays below 2^30
    // The bytes of v + 0x808080, the lower three less 128 each, are the digits.  The sum is made in float32 (0x808080 has its 8 leading bits only).
    uint32_t z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = (uint32_t)(int)__builtin_fmaf(v[e], up, 8421504.0f);
    uint32_t a[4][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {                              // bytes of 4 columns by digit
        const uint32_t p0 = byte_perm(z[4 * h + 1], z[4 * h], 0x05010400u), p1 = byte_perm(z[4 * h + 1], z[4 * h], 0x07030602u);
        const uint32_t q0 = byte_perm(z[4 * h + 3], z[4 * h + 2], 0x05010400u), q1 = byte_perm(z[4 * h + 3], z[4 * h + 2], 0x07030602u);
        a[0][h] = byte_perm(q0, p0, 0x05040100u) ^ 0x80808080u;
        a[1][h] = byte_perm(q0, p0, 0x07060302u) ^ 0x80808080u;
        a[2][h] = byte_perm(q1, p1, 0x05040100u) ^ 0x80808080u;
        a[3][h] = byte_perm(q1, p1, 0x07060302u);
    }
    const bool odd = threadIdx.x & 1, upper = threadIdx.x & 2;
#pragma unroll
    for (int h = 0; h < 2; ++h) {                              // 4 x 4 transpose over the lanes t of a row
#pragma unroll
        for (int d = 0; d < 4; d += 2) {
            const uint32_t x = lane_xor<1>(a[d + 1][h]), y = lane_xor<1>(a[d][h]);
            a[d][h] = odd ? x : a[d][h];
            a[d + 1][h] = odd ? a[d + 1][h] : y;
        }
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const uint32_t x = lane_xor<2>(a[d + 2][h]), y = lane_xor<2>(a[d][h]);
            a[d][h] = upper ? x : a[d][h];
            a[d + 2][h] = upper ? a[d + 2][h] : y;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) { B[2 * j] = a[j][0]; B[2 * j + 1] = a[j][1]; }
}

// the sums of 16 q * v from those of its digits
__device__ __forceinline__ float join_digits(const i32x4_t &d) {
    return __builtin_fmaf((float)((d[3] << 8) + d[2]), 65536.0f, (float)((d[1] << 8) + d[0]));
}

template <int G>
struct Q4Words {                                               // a lane's part of a block: 32 weights of a row and the row's scales
    static constexpr int per = kQ4Block / G;
    uint4 w;
    uint32_t s[(per + 1) / 2];
    template <bool ONCE>                                       // read by nobody else
    __device__ __forceinline__ void load(const Q4Kernel &a, size_t block, int lane) {
        typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;
        const u32x4_t *src = reinterpret_cast<const u32x4_t *>(a.W) + block * 64 + lane;
        const u32x4_t v = ONCE ? __builtin_nontemporal_load(src) : *src;
        w = uint4{v.x, v.y, v.z, v.w};
        const uint16_t *p = a.S + (block * 16 + (lane & 15)) * per;
        if constexpr (G == 128) s[0] = *p;
        else if constexpr (G == 64) s[0] = *reinterpret_cast<const uint32_t *>(p);
        else { const uint2 q = *reinterpret_cast<const uint2 *>(p); s[0] = q.x; s[1] = q.y; }
    }
    __device__ __forceinline__ float scale(int i) const { return i & 1 ? bf16_hi(s[i / 2]) : bf16_lo(s[i / 2]); }
    // operand of step s
    __device__ __forceinline__ i32x4_t operand(int i) const {
        const uint32_t a = i ? w.z : w.x, b = i ? w.w : w.y;
        return i32x4_t{(int)(a & 0xf0f0f0f0u), (int)((a << 4) & 0xf0f0f0f0u), (int)(b & 0xf0f0f0f0u), (int)((b << 4) & 0xf0f0f0f0u)};
    }
};

// The digits' sums of each group of a block: digits x, weights w, two steps of 64 columns
template <int G>
__device__ __forceinline__ void group_sums(const i32x4_t (&x)[2], const i32x4_t (&w)[2], i32x4_t (&o)[kQ4Block / G]) {
    const i32x4_t none = {0, 0, 0, 0};
    auto half = [](const i32x4_t &v, int h) { return (long)((unsigned long)(unsigned)v[2 * h + 1] << 32 | (unsigned)v[2 * h]); };
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if constexpr (G == 32) {
            o[2 * s] = __builtin_amdgcn_mfma_i32_16x16x32_i8(half(x[s], 0), half(w[s], 0), none, 0, 0, 0);
            o[2 * s + 1] = __builtin_amdgcn_mfma_i32_16x16x32_i8(half(x[s], 1), half(w[s], 1), none, 0, 0, 0);
        } else if constexpr (G == 64) {
            o[s] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[s], w[s], none, 0, 0, 0);
        } else {
            o[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[s], w[s], s ? o[0] : none, 0, 0, 0);
        }
    }
}

// The value (gate, up: of the two halves of a tile) of row `row`, column n of tile t into place; the 16 columns of a row sit in 16 neighbouring lanes
__device__ __forceinline__ void finish(const Q4Kernel &a, bool active, int row, int t, int n, float sum, float up, float inv) {
    const int col = t * 16 + n;
    if (a.epilogue == EPI_SWIGLU) {
        if (!active || n >= 8) return;
        const float gate = sum * inv;
        a.Xout[(size_t)row * a.K_out + t * 8 + n] = gate / (1.0f + expf(-gate)) * (up * inv);
    } else if (a.epilogue == EPI_STORE) {
        if (active && col < a.N) a.Y[(size_t)row * a.ldy + col] = sum * inv;
    } else {
        float hnew = 0.f;
        if (active) {
            hnew = a.Y[(size_t)row * a.ldy + col] + sum;
            a.Y[(size_t)row * a.ldy + col] = hnew;
            if (a.gain_next) a.Xnext[(size_t)row * a.N + col] = hnew * a.gain_next[col];
        }
        const float sq = row_sum(hnew * hnew);
        if (a.ssq_out && n == 0 && active) a.ssq_out[(size_t)row * a.tiles + t] = sq;
    }
}

// 1 / rms of rows row0 .. last - 1 into inv_s (1 without a norm); the caller synchronises
template <int WAVES>
__device__ __forceinline__ void row_scales(const Q4Kernel &a, int last, float *inv_s) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (a.ssq_in) {
        const int parts = a.ssq_in_parts;
        for (int r = a.row0 + w; r < last; r += WAVES) {
            const float *part = a.ssq_in + (size_t)r * (a.K / 16);
            float v[4], sum = 0.f;                             // 256 parts (K = 4096) in one look
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = lane + 64 * i < parts ? part[lane + 64 * i] : 0.f;
            for (int p = lane + 256; p < parts; p += 64) sum += part[p];
            sum = wave_sum(((v[0] + v[1]) + (v[2] + v[3])) + sum);
            if (lane == 0) inv_s[r] = 1.0f / sqrtf(sum * a.inv_d + a.eps);
        }
    } else if (threadIdx.x < kMaxRows) {
        inv_s[threadIdx.x] = 1.0f;
    }
}

// ---- few rows (1 .. 16): the waves of a workgroup share a tile's blocks ------------------------------------
// A workgroup takes tiles of 16 outputs; its waves take the blocks of a tile's row in units of NB and meet in LDS.  Every workgroup makes
// the digits for itself, while its first weights are on their way.  KEEP: one unit per wave covers K; its digits stay in
// registers for all of the workgroup's tiles, and a block's words are replaced by the next tile's as soon as they
// are used.  Otherwise any K, and the digits of a unit are made anew for every tile.
// Rows: FULL groups of up to 4 and (SINGLE) one row more.  A row group's digits take as long to make for one row as for four, so the single
// row's are made for NB blocks at once, in the places of the group's other rows: the matrix core then multiplies a block's weights by the digits
// of all NB blocks, and of the sums only the lanes of the right block's place are added.
// Bound by the stream of weights, and where that is short by a workgroup's chain: first loads, digits, products, sums through LDS.  G = 128: 22016 x 4096 one
// row 10.4 us (46.9 MB, 4.5 TB/s), 5 rows 12.1, 8 rows 13.5, 12 rows 18; 4096 x 4096 one row 4.9 (4.1 where the weights are in the caches); 768 x 768 3.0, of which an empty kernel is most.
template <int WAVES, int FULL, bool SINGLE, int G, int NB, bool KEEP>
__global__ __launch_bounds__(WAVES * 64) void q4_few_kernel(Q4Kernel a) {
    constexpr int NG = FULL + SINGLE, per = kQ4Block / G, GROUPS = FULL > 0 ? FULL : 1;
    // Whether the words behind the last tile's are left unread, or (a loop without that branch) the last tile's are read twice.  Branch / read twice:
    // one row, 12288 x 8192 10.1 / 11.3 us; 5 rows, the same 14.7 / 15.4, 22016 x 4096 12.6 / 12.4; 12 rows, 22016 x 4096 18.4 / 17.8.  (5 rows at G = 32: 118 registers would go to memory.)
    constexpr bool STOP = FULL == 0 || (FULL == 1 && NB == 4 && G == 128);
    static_assert(NB <= kQ4Rows, "places of the single row's blocks");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, t = lane & 3, c = (lane & 15) >> 2;
    __shared__ float red[2][WAVES][NG][64];                    // [..][activation row][16 outputs]
    __shared__ float inv_s[kMaxRows];
    Q4Words<G> words[NB];
    i32x4_t B[GROUPS][NB][2], B1[2];
    float f[GROUPS][NB], f1[NB];                               // of the row whose sums the lane gets
    auto load_words = [&](int tile, int b, Q4Words<G> &o) __attribute__((always_inline)) { o.template load<true>(a, (size_t)tile * a.KB + min(b, a.KB - 1), lane); };
    auto convert = [&](const float (&v)[8], i32x4_t (&o)[2]) __attribute__((always_inline)) {
        const int e = block_exponent(v);
        uint32_t d[8];
        block_digits(v, e, d);
        o[0] = i32x4_t{(int)d[0], (int)d[1], (int)d[2], (int)d[3]};
        o[1] = i32x4_t{(int)d[4], (int)d[5], (int)d[6], (int)d[7]};
        return digit_factor(__shfl(e, 4 * g, 64));
    };
    // digits of blocks b0 .. b0 + NB - 1 (beyond the matrix: zeros)
    auto digits = [&](int b0) __attribute__((always_inline)) {
        auto first = [&](int b) __attribute__((always_inline)) { return b < a.KB ? kQ4Block * b + 32 * t + 8 * g : a.K; };
        float v1[8];
#pragma unroll
        for (int r0 = 0; r0 < (FULL > 0 ? FULL : 1); r0 += 2) {    // two groups at a time: what their loads take of registers
            float v[2][NB][8];
            with_kind(a, [&](auto kind) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int rg = r0; rg < FULL && rg < r0 + 2; ++rg) load_x8<kind()>(a, a.row0 + kQ4Rows * rg + c, first(b0 + i), v[rg - r0][i]);
                if (SINGLE && r0 == 0) load_x8<kind()>(a, a.row0 + kQ4Rows * FULL, c < NB ? first(b0 + c) : a.K, v1);
            });
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int rg = r0; rg < FULL && rg < r0 + 2; ++rg) f[rg][i] = convert(v[rg - r0][i], B[rg][i]);
        }
        if (SINGLE) {
            const float own = convert(v1, B1);
#pragma unroll
            for (int i = 0; i < NB; ++i) f1[i] = g == i ? own : 0.f;
        }
    };
    float sum[NG];
    auto multiply = [&](int i) __attribute__((always_inline)) {
        const i32x4_t x[2] = {words[i].operand(0), words[i].operand(1)};
        float sc[per];
#pragma unroll
        for (int p = 0; p < per; ++p) sc[p] = words[i].scale(p) * kQ4ScaleDown;
#pragma unroll
        for (int rg = 0; rg < NG; ++rg) {
            const bool single = rg == FULL;
            const float factor = single ? f1[i] : f[single ? 0 : rg][i];
            i32x4_t o[per];
            group_sums<G>(single ? B1 : B[single ? 0 : rg][i], x, o);
            float block = join_digits(o[0]) * sc[0];
#pragma unroll
            for (int p = 1; p < per; ++p) block = __builtin_fmaf(join_digits(o[p]), sc[p], block);
            sum[rg] = __builtin_fmaf(block, factor, sum[rg]);
        }
    };
    int tile = blockIdx.x;
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < NB; ++i) load_words(tile, w * NB + i, words[i]);
        digits(w * NB);
    }
    row_scales<WAVES>(a, min(a.rows, a.row0 + NG * kQ4Rows), inv_s);
    int parity = 0;
    for (; tile < a.tiles; tile += gridDim.x, parity ^= 1) {
#pragma unroll
        for (int rg = 0; rg < NG; ++rg) sum[rg] = 0.f;
        if (KEEP) {
            const bool more = tile + (int)gridDim.x < a.tiles;
            const int next = more ? tile + (int)gridDim.x : tile;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                multiply(i);
                if (!STOP || more) load_words(next, w * NB + i, words[i]);
                __builtin_amdgcn_sched_barrier(0);            // keep "use, replace" in program order
            }
        } else {
            for (int b0 = w * NB; b0 < a.KB; b0 += WAVES * NB) {
#pragma unroll
                for (int i = 0; i < NB; ++i) load_words(tile, b0 + i, words[i]);
                digits(b0);
#pragma unroll
                for (int i = 0; i < NB; ++i) multiply(i);
            }
        }
        if (SINGLE) sum[FULL] = xor_reduce<32, 16>(sum[FULL], AddOp());       // (its row is the first place's; the others hold no row)
#pragma unroll
        for (int rg = 0; rg < NG; ++rg) red[parity][w][rg][lane] = sum[rg];
        __syncthreads();
        for (int e = threadIdx.x; e < NG * 64; e += WAVES * 64) {
            const int n = e & 15, i = e & 63, rg = e >> 6, row = a.row0 + kQ4Rows * rg + (i >> 4);
            float s = 0.f, up = 0.f;
#pragma unroll
            for (int ww = 0; ww < WAVES; ++ww) s += red[parity][ww][rg][i];
            if (a.epilogue == EPI_SWIGLU)
#pragma unroll
                for (int ww = 0; ww < WAVES; ++ww) up += red[parity][ww][rg][i ^ 8];
            finish(a, row < a.rows, row, tile, n, s, up, inv_s[row < a.rows ? row : 0]);
        }
        // no second barrier: the next tile writes the other half of `red`
    }
}

// ---- many rows -------------------------------------------------------------------------------
// The digits are made once, by a kernel of their own: a wave per row group and chunk of 4 blocks (more where K is over 16384, so that there are
// at most 32), whose values of a row share an exponent.  40 x 4096 4.6 us, a kernel's start and one round trip (an exponent per block of 128, as the
// kernel of few rows has, took a multiplication per sum more in the product).  Layout: [row group][block][step][lane] of 16 bytes, then the factors [row group][chunk][row].
constexpr int kQ4Chunks = 32;
static int chunk_shift(int KB) {
    int s = 2;
    while ((KB + (1 << s) - 1) >> s > kQ4Chunks) ++s;
    return s;
}
template <bool KEEP>                                           // the chunk's values stay in registers between the search for the largest magnitude and the digits
__global__ __launch_bounds__(64) void q4_digits_kernel(Q4Kernel a, uint4 *digits, float *factors, int shift) {
    const int chunks = (a.KB + (1 << shift) - 1) >> shift, rg = blockIdx.x / chunks, chunk = blockIdx.x - rg * chunks;
    const int lane = threadIdx.x, g = lane >> 4, t = lane & 3, c = (lane & 15) >> 2;
    const int b0 = chunk << shift, n = min(1 << shift, a.KB - b0);
    float m = 0.f, v[KEEP ? 4 : 1][8];
    auto load = [&](auto kind, int i, float (&x)[8]) __attribute__((always_inline)) { load_x8<kind()>(a, kQ4Rows * rg + c, i < n ? kQ4Block * (b0 + i) + 32 * t + 8 * g : a.K, x); };
    auto look = [&](const float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m = __builtin_elementwise_maximum(m, fabsf(x[e]));
    };
    with_kind(a, [&](auto kind) __attribute__((always_inline)) {
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load(kind, i, v[KEEP ? i : 0]);
        } else {
            for (int i = 0; i < n; ++i) { load(kind, i, v[0]); look(v[0]); }
        }
    });
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) look(v[KEEP ? i : 0]);
    }
    const int exponent = shared_exponent(m);
    if (g == 0 && t == 0) factors[(rg * chunks + chunk) * kQ4Rows + c] = digit_factor(exponent);
    auto make = [&](int i, const float (&x)[8]) __attribute__((always_inline)) {
        uint32_t B[8];
        block_digits(x, exponent, B);
        if (i >= n) return;
        uint4 *dst = digits + ((size_t)rg * a.KB + b0 + i) * 128 + lane;
        dst[0] = uint4{B[0], B[1], B[2], B[3]};
        dst[64] = uint4{B[4], B[5], B[6], B[7]};
    };
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) make(i, v[KEEP ? i : 0]);
    } else {
        with_kind(a, [&](auto kind) __attribute__((always_inline)) {
            for (int i = 0; i < n; ++i) { load(kind, i, v[0]); make(i, v[0]); }
        });
    }
}

// sum[i][rg] += a block of tile i of a pair times the digits of NG row groups at src (LDS).  Written out in the order in which it should be
// issued: digits are asked for two row groups ahead, and while the matrix core has a row group the sums of the one before are added (LAG; not
// where four sums a row group in two sets take too many registers: 64 rows x 32000 x 4096 at G = 32 102 us with spills, 73 without).
template <int NG, int G>
__device__ __forceinline__ void pair_products(const Q4Words<G> (&words)[2], const uint4 *src, float (&sum)[2][NG]) {
    constexpr int per = kQ4Block / G, AHEAD = 2, LAG = G == 32 && NG >= 12 ? 0 : 1;
    uint4 B[AHEAD + 1][2];
    auto ask = [&](int rg) __attribute__((always_inline)) { B[rg % (AHEAD + 1)][0] = src[rg * 128]; B[rg % (AHEAD + 1)][1] = src[rg * 128 + 64]; };
#pragma unroll
    for (int rg = 0; rg < (AHEAD < NG ? AHEAD : NG); ++rg) ask(rg);
    i32x4_t x[2][2], acc[1 + LAG][2][per];
    float sc[2][per];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i][0] = words[i].operand(0); x[i][1] = words[i].operand(1);
#pragma unroll
        for (int p = 0; p < per; ++p) sc[i][p] = words[i].scale(p) * kQ4ScaleDown;
    }
#pragma unroll
    for (int rg = 0; rg < NG + LAG; ++rg) {
        if (rg + AHEAD < NG) ask(rg + AHEAD);
        if (rg < NG) {
            const i32x4_t d[2] = {__builtin_bit_cast(i32x4_t, B[rg % (AHEAD + 1)][0]), __builtin_bit_cast(i32x4_t, B[rg % (AHEAD + 1)][1])};
#pragma unroll
            for (int i = 0; i < 2; ++i) group_sums<G>(d, x[i], acc[rg & LAG][i]);
        }
        if (rg >= LAG) {
            const int done = rg - LAG;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int p = 0; p < per; ++p) sum[i][done] = __builtin_fmaf(join_digits(acc[done & LAG][i][p]), sc[i][p], sum[i][done]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// 8 multiplying waves, 4 pairs of tiles x even and odd blocks, and 4 loader waves that bring the digits of two blocks after
// the other into LDS (LDS-direct loads, NBUF - 1 steps ahead), where a multiplying wave uses what it reads for both of its tiles.  The
// weights come through registers, RD steps ahead.  To fill the chip where a matrix has few tiles the blocks are cut
// into `slices` across workgroups, whose sums q4_join_kernel adds.  (Workgroups that
// begin at different steps of their slice, as the batched projections in bf16 do, are 1 to 2 % slower here, and weights loaded non-temporally 4 %.)
// 40 rows x 32000 x 4096 at G = 128 29.6 us (72 MB, 2.4 TB/s), 64 rows x 11003 x 4099 at G = 64 27.  By counters, of the cycles of a busy SIMD there: products 35 and 30 %, other
// vector instructions 44 and 61 (5.1 and 8.2 a product, where the joining of the sums takes 3 and 6: the rest are the masks of the weights, scales, addresses), both at
// once 14 and 11, neither 35 and 20: two multiplying waves a SIMD that wait at the same barriers.  LDS reads take a fifth of a CU's cycles, without conflicts.  (Four products
// and twelve other instructions take a SIMD 42.7 ns in a loop of nothing else, where the products alone take 31.9 and the others 22.2.)
constexpr int kQ4ManyTiles = 8, kQ4Loaders = 4, kQ4MaxSlices = 8;
constexpr int many_ring(int NG, int G) { return G == 32 && NG >= 8 ? 2 : NG == 16 ? 3 : 4; }     // what registers allow
constexpr int many_buffers(int NG) { return NG <= 8 ? 4 : NG <= 12 ? 3 : 2; }
template <int NG, int G>
__global__ __launch_bounds__((8 + kQ4Loaders) * 64) __attribute__((amdgpu_waves_per_eu(2, 3))) void q4_many_kernel(Q4Kernel a, const uint4 *digits, const float *factors, float *partials, int slices, int ng, int shift) {
    constexpr int RD = many_ring(NG, G), NBUF = many_buffers(NG), PB = 4 * NG / kQ4Loaders;      // pieces of 1 KiB per loader wave and step
    static_assert((NBUF - 1) * PB <= 63, "outstanding loads of a loader wave");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), odd = w >> 2, wt = w & 3;
    const int group = blockIdx.x / slices, slice = blockIdx.x - group * slices;
    const int b0 = (int)((long)a.KB * slice / slices), len = (int)((long)a.KB * (slice + 1) / slices) - b0;
    const int steps = (len + 1) / 2;                           // (those beyond load what is never used)
    extern __shared__ uint4 lds[];                             // [NBUF][even, odd][NG][2][64]
    __shared__ float inv_s[kMaxRows];
    __shared__ float F[kQ4Chunks][kMaxRows];                   // factors of the digits
    const int chunks = (a.KB + (1 << shift) - 1) >> shift;
    for (int e = threadIdx.x; e < chunks * ng * kQ4Rows; e += (8 + kQ4Loaders) * 64) {
        const int rg = e / (chunks * kQ4Rows), in = e - rg * chunks * kQ4Rows;
        F[in / kQ4Rows][rg * kQ4Rows + (in & 3)] = factors[e];
    }
    float sum[2][NG], total[2][NG];                            // of a chunk, of all
    const int t0 = group * kQ4ManyTiles + 2 * wt;
    if (w >= 8) {
        const int first = w - 8, o = first >> 1;               // two loaders for the even blocks, two for the odd ones
        unsigned offset[PB];                                   // bytes from the block's first row group: a handful of scalar instructions per load
#pragma unroll
        for (int r = 0; r < PB; ++r) {
            const int piece = (first & 1) + 2 * r;             // of the block's 2 NG
            offset[r] = (unsigned)(min(piece >> 1, ng - 1) * a.KB * 128 + (piece & 1) * 64) * 16u;
        }
        int buffer = 0;
        auto issue = [&](int s) __attribute__((always_inline)) {
            const char *src = reinterpret_cast<const char *>(digits) + (size_t)(b0 + min(2 * s + o, len - 1)) * 2048;
            uint4 *dst = lds + (buffer * 2 + o) * NG * 128 + (first & 1) * 64;
#pragma unroll
            for (int r = 0; r < PB; ++r)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + offset[r] + 16u * lane),
                                                 (__attribute__((address_space(3))) void *)(dst + r * 128), 16, 0, 0);
            buffer = buffer + 1 == NBUF ? 0 : buffer + 1;
        };
#pragma unroll
        for (int s = 0; s < NBUF - 1; ++s) issue(s);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NBUF - 2) * PB) : "memory");   // step 0 has landed (loads complete in order), and what this wave wrote to F
        __builtin_amdgcn_s_barrier();
        for (int s = 0; s < steps; ++s) {
            issue(s + NBUF - 1);                               // into the buffer that the products left one step ago
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NBUF - 2) * PB) : "memory");   // step s + 1 has landed
            __builtin_amdgcn_s_barrier();
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int rg = 0; rg < NG; ++rg) sum[i][rg] = total[i][rg] = 0.f;
        Q4Words<G> ring[RD][2];
        auto weights = [&](int slot, int s) __attribute__((always_inline)) {
            const int b = b0 + min(2 * s + odd, len - 1);
#pragma unroll
            for (int i = 0; i < 2; ++i) ring[slot][i].template load<false>(a, (size_t)min(t0 + i, a.tiles - 1) * a.KB + b, lane);     // (beyond the matrix: a valid tile, dropped)
        };
#pragma unroll
        for (int s = 0; s < RD; ++s) weights(s, s);
        __syncthreads();
        int buffer = 0, chunk = (b0 + min(odd, len - 1)) >> shift;
        auto chunk_done = [&] __attribute__((always_inline)) {
            const float *f = &F[chunk][lane >> 4];
#pragma unroll
            for (int rg = 0; rg < NG; ++rg) {
                const float factor = f[rg * kQ4Rows];          // (row groups that there are not: never used)
#pragma unroll
                for (int i = 0; i < 2; ++i) { total[i][rg] = __builtin_fmaf(sum[i][rg], factor, total[i][rg]); sum[i][rg] = 0.f; }
            }
        };
        for (int s0 = 0; s0 < steps; s0 += RD) {
#pragma unroll
            for (int h = 0; h < RD; ++h) {
                if (s0 + h >= steps) break;
                const int p = 2 * (s0 + h) + odd;               // block of the slice
                if (p < len) {
                    if ((b0 + p) >> shift != chunk) {
                        chunk_done();
                        chunk = (b0 + p) >> shift;
                    }
                    pair_products<NG, G>(ring[h], lds + (buffer * 2 + odd) * NG * 128 + lane, sum);
                }
                weights(h, s0 + h + RD);
                __builtin_amdgcn_sched_barrier(0);             // keep "multiply, refill the freed slots" in program order
                buffer = buffer + 1 == NBUF ? 0 : buffer + 1;
                __syncthreads();
            }
        }
        chunk_done();
    }
    __syncthreads();                                           // the loaders' surplus steps have landed: the buffers are free
    float *red = reinterpret_cast<float *>(lds);               // [even, odd][tile of the group][NG][activation row][16 outputs]
    constexpr int HALF = kQ4ManyTiles * NG * 64;
    if (w < 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int rg = 0; rg < NG; ++rg) red[odd * HALF + ((2 * wt + i) * NG + rg) * 64 + lane] = total[i][rg];
    }
    row_scales<8 + kQ4Loaders>(a, a.rows, inv_s);
    __syncthreads();
    for (int e = threadIdx.x; e < HALF; e += (8 + kQ4Loaders) * 64) {
        const int n = e & 15, rg = (e >> 6) % NG, row = kQ4Rows * rg + ((e >> 4) & 3), tile = group * kQ4ManyTiles + (e >> 6) / NG;
        const bool active = row < a.rows && tile < a.tiles;
        const float s = red[e] + red[HALF + e], up = red[e ^ 8] + red[HALF + (e ^ 8)];
        if (slices > 1) {
            if (active) partials[((size_t)slice * a.rows + row) * ((size_t)a.tiles * 16) + tile * 16 + n] = s;
        } else {
            finish(a, active, row, tile, n, s, up, inv_s[active ? row : 0]);
        }
    }
}

// The sums of the slices, in order, into place: 16 rows of a tile per workgroup.  4.8 us for 40 x 4096 in 8 slices: a kernel's start, one round trip.  (The last workgroup
// of a tile group to arrive reading the others' sums instead: 64 rows x 11003 x 4099 41 us became 44.)
__global__ __launch_bounds__(256) void q4_join_kernel(Q4Kernel a, const float *partials, int slices) {
    const int tile = blockIdx.x, n = threadIdx.x & 15, row = blockIdx.y * 16 + (threadIdx.x >> 4);
    __shared__ float inv_s[kMaxRows];
    const bool active = row < a.rows;
    const size_t ld = (size_t)a.tiles * 16;
    float part[kQ4MaxSlices];                                  // all on their way together
#pragma unroll
    for (int i = 0; i < kQ4MaxSlices; ++i) part[i] = active && i < slices ? partials[((size_t)i * a.rows + row) * ld + tile * 16 + n] : 0.f;
    a.row0 = blockIdx.y * 16;
    row_scales<4>(a, min(a.rows, a.row0 + 16), inv_s);
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kQ4MaxSlices; ++i) s += part[i];
    finish(a, active, row, tile, n, s, lane_xor<8>(s), inv_s[active ? row : 0]);
}

// Up to how many rows the kernel of few rows goes: as many row groups as a workgroup's registers keep the digits of, or, made anew for each of a
// workgroup's tiles, as many as pay.  Few / many at G = 128, us: 16 rows, 768 x 768 6.1 / 9.4; 12 rows, 4096 x 4096 12.2 / 16.1, 32000 x 4096 20.9 / 22.5;
// one tile each: 8 rows, 4096 x 8192 13.3 / 14.5, 4096 x 11008 15.7 / 15.7, 4096 x 16384 21.4 / 16.8, 4 rows there 15.1 / 16.8;
// more tiles: 8 rows, 12288 x 8192 33.9 / 23.9, 5 rows there 14.7 / 23.8; 4 rows, 8192 x 11008 19.9 / 19.0, 2 rows 17.0 / 18.8, 32000 x 11008 60.8 / 45.0 (one row 39.0 / 45).
static int few_rows(int N, int K) {
    const int KB = (K + kQ4Block - 1) / kQ4Block, rounds = ((N + 15) / 16 + 255) / 256;
    if (KB <= 32) return KB <= 16 ? 16 : 12;
    if (rounds == 1) return KB <= 96 ? 8 : 4;
    return KB <= 64 ? 5 : rounds == 2 ? 3 : 1;
}
// Slices of K: what makes rounds of workgroups x blocks of one the least, with about 4 blocks' time for a workgroup's start and end.  (Where neither one nor more
// slices fill the chip evenly some of it idles: 22016 x 4096 is 172 workgroups, 29 us at 40 rows.)
static int many_slices(int N, int K) {
    const int groups = ((N + 15) / 16 + kQ4ManyTiles - 1) / kQ4ManyTiles, KB = (K + kQ4Block - 1) / kQ4Block;
    int best = 1;
    long least = 0;
    for (int s = 1; s <= std::min(kQ4MaxSlices, std::max(1, KB / 4)); ++s) {
        const long cost = (long)((groups * s + 255) / 256) * ((KB + s - 1) / s + 4);
        if (s == 1 || cost < least) { best = s; least = cost; }
    }
    return best;
}
static size_t digit_bytes(int rows, int K) { return (size_t)((rows + 3) / 4) * ((K + kQ4Block - 1) / kQ4Block) * 2048; }

size_t q4_workspace_bytes(int rows, int N, int K) {
    if (rows <= few_rows(N, K)) return 0;
    const int slices = many_slices(N, K);
    return digit_bytes(rows, K) + kQ4Chunks * kMaxRows * 4 + (slices > 1 ? (size_t)slices * rows * ((N + 15) / 16 * 16) * 4 : 0);
}

template <int NG, int G>
static hipError_t launch_many(const Q4Kernel &k, const uint4 *digits, const float *factors, float *partials, int slices, int ng, int shift, hipStream_t stream) {
    constexpr size_t lds = (size_t)many_buffers(NG) * NG * 4096;
    const hipError_t ready = hipFuncSetAttribute((const void *)q4_many_kernel<NG, G>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (ready != hipSuccess) return ready;
    const int groups = (k.tiles + kQ4ManyTiles - 1) / kQ4ManyTiles;
    hipLaunchKernelGGL((q4_many_kernel<NG, G>), dim3(groups * slices), dim3((8 + kQ4Loaders) * 64), lds, stream, k, digits, factors, partials, slices, ng, shift);
    return hipGetLastError();
}

// Workgroups: one per CU, two where they are small (K of at most 8 blocks), each with as many tiles as that leaves it, so that digits are made
// once a CU (twice as many: 5 rows, 8192 x 2048 7.1 us, now 6.0; 16384 x 1024 7.3, now 6.3; one row, 16384 x 2048 5.9, now 6.1).  Blocks of K per wave: 1 up to 8 (4 rows, 768 x 768
// 3.1 us, with two 3.3), 2 up to 32 (16 waves of 2 and 8 of 4, 12288 x 4096: one row 7.2 / 7.0, 4 rows 8.4 / 9.7, 5 rows 9.3 / 14.4), 4 beyond.  Digits that stay
// pay where a workgroup has a second tile (5 rows, 12288 x 8192 15.3 us, made anew 26.0; 4096 x 8192, one tile each, 10.6 and 9.8).
template <int FULL, bool SINGLE, int G>
static void launch_few(const Q4Kernel &k, hipStream_t stream) {
    const int KB = k.KB;
    if constexpr (FULL > 2) {                                  // (K of at most 32 blocks, 16 for four groups: see few_rows)
        if (FULL == 4 || KB <= 16) hipLaunchKernelGGL((q4_few_kernel<8, FULL, SINGLE, G, 2, true>), dim3(std::min(k.tiles, 256)), dim3(512), 0, stream, k);
        else if constexpr (FULL == 3) hipLaunchKernelGGL((q4_few_kernel<8, FULL, SINGLE, G, 4, true>), dim3(std::min(k.tiles, 256)), dim3(512), 0, stream, k);
    } else if (KB <= 8) hipLaunchKernelGGL((q4_few_kernel<8, FULL, SINGLE, G, 1, true>), dim3(std::min(k.tiles, 512)), dim3(512), 0, stream, k);
    else if (KB <= 16) hipLaunchKernelGGL((q4_few_kernel<8, FULL, SINGLE, G, 2, true>), dim3(std::min(k.tiles, 256)), dim3(512), 0, stream, k);
    else if (KB <= 32) hipLaunchKernelGGL((q4_few_kernel<16, FULL, SINGLE, G, 2, true>), dim3(std::min(k.tiles, 256)), dim3(1024), 0, stream, k);
    else if constexpr (FULL == 2) hipLaunchKernelGGL((q4_few_kernel<16, FULL, SINGLE, G, 2, false>), dim3(std::min(k.tiles, 256)), dim3(1024), 0, stream, k);   // (registers)
    else if (KB <= 64 && k.tiles > 256) hipLaunchKernelGGL((q4_few_kernel<16, FULL, SINGLE, G, 4, true>), dim3(std::min(k.tiles, 256)), dim3(1024), 0, stream, k);
    else hipLaunchKernelGGL((q4_few_kernel<16, FULL, SINGLE, G, 4, false>), dim3(std::min(k.tiles, 256)), dim3(1024), 0, stream, k);
}

hipError_t launch_q4_gemm(const Q4GemmArgs &a, int epilogue, hipStream_t stream) {
    if (a.rows < 1 || a.rows > kMaxRows || !q4_group_ok(a.group)) return hipErrorInvalidValue;
    Q4Kernel k{};
    k.W = (const uint4 *)a.W;
    k.S = (const uint16_t *)((const char *)a.W + q4_scales_offset(a.N, a.K));
    k.N = a.N; k.K = a.K; k.KB = (a.K + kQ4Block - 1) / kQ4Block; k.tiles = (a.N + 15) / 16;
    k.X = a.X; k.x_kind = a.x_kind; k.ldx = a.ldx; k.KS = (a.K + 31) / 32; k.rows = a.rows;
    k.Y = a.Y; k.ldy = a.ldy;
    k.ssq_in = a.ssq_in; k.ssq_in_parts = a.ssq_in_parts; k.inv_d = 1.0f / (float)a.K; k.eps = a.eps;
    k.gain_next = a.gain_next; k.Xnext = a.Xnext; k.ssq_out = a.ssq_out;
    k.Xout = a.Xout; k.K_out = a.K_out; k.epilogue = epilogue;
    hipError_t rc = hipSuccess;
    const hipError_t launched = with_group(a.group, [&](auto g) {
        const int few = few_rows(a.N, a.K);
        if (a.rows == 1) launch_few<0, true, g()>(k, stream);
        else if (a.rows > few) {
            const int ng = (a.rows + kQ4Rows - 1) / kQ4Rows, slices = many_slices(a.N, a.K);
            uint4 *digits = (uint4 *)a.workspace;
            float *factors = (float *)((char *)a.workspace + digit_bytes(a.rows, a.K)), *partials = factors + kQ4Chunks * kMaxRows;
            const int shift = chunk_shift(k.KB), chunks = (k.KB + (1 << shift) - 1) >> shift;
            if (shift == 2) hipLaunchKernelGGL(q4_digits_kernel<true>, dim3(ng * chunks), dim3(64), 0, stream, k, digits, factors, shift);
            else hipLaunchKernelGGL(q4_digits_kernel<false>, dim3(ng * chunks), dim3(64), 0, stream, k, digits, factors, shift);
            if (ng <= 4) rc = launch_many<4, g()>(k, digits, factors, partials, slices, ng, shift, stream);
            else if (ng <= 6) rc = launch_many<6, g()>(k, digits, factors, partials, slices, ng, shift, stream);
            else if (ng <= 8) rc = launch_many<8, g()>(k, digits, factors, partials, slices, ng, shift, stream);
            else if (ng <= 10) rc = launch_many<10, g()>(k, digits, factors, partials, slices, ng, shift, stream);
            else if (ng <= 12) rc = launch_many<12, g()>(k, digits, factors, partials, slices, ng, shift, stream);
            else rc = launch_many<16, g()>(k, digits, factors, partials, slices, ng, shift, stream);
            if (rc == hipSuccess && slices > 1) hipLaunchKernelGGL(q4_join_kernel, dim3(k.tiles, (a.rows + 15) / 16), dim3(256), 0, stream, k, partials, slices);
        } else if (a.rows <= kQ4Rows) launch_few<1, false, g()>(k, stream);
        else if (a.rows == kQ4Rows + 1) launch_few<1, true, g()>(k, stream);
        else if (a.rows <= 2 * kQ4Rows) launch_few<2, false, g()>(k, stream);
        else if (a.rows <= 3 * kQ4Rows) launch_few<3, false, g()>(k, stream);
        else launch_few<4, false, g()>(k, stream);
    });
    return rc != hipSuccess ? rc : launched;
}

}  // namespace spd
