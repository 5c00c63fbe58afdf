// Projections with weights and activations in 8-bit floating point (4 exponent and 3 mantissa bits) and a power-of-two scale per
// block of 128:  x = 2^e q,  e the smallest integer with max|x| <= 448 2^e over the block (448 is the format's largest value), q
// rounded to nearest even.  Weights have a scale per 128 rows and 128 columns, activations one per row and 128 columns.
//   y[m, n] = sum over blocks b of 2^(ex[m, b] + ew[n / 128, b]) sum over k in b of qx[m, k] qw[n, k]
// The matrix instruction of 16 x 16 x 128 8-bit operands takes both exponents per operand row and multiplies them in, so a block is one
// instruction with nothing beside it, and sums stay in its fp32 accumulators.  It does not keep all bits of a block's smaller products
// (5e-6 of the result's norm on values of a normal distribution, 5e-5 on values of every exponent): nothing beside a bf16 result's own 2^-9, and it
// serves those.  For fp32 results the 8-bit values are widened to bf16 (exactly) and multiplied by the bf16 instructions, whose sums are fp32
// throughout, at half the rate; a block's sum is then scaled and added.
//
// Layout of both operands, [rows, k]: tiles of 16 rows, per tile and block of 128 columns 2 KiB: piece (half, g, r) of 16 bytes
// holds row r, columns half * 64 + g * 16 ..; lane g * 16 + r of a wave loads the pieces of both halves, 1 KiB per instruction.
// (The instruction would have 32 consecutive columns in a lane; any order does that both operands share.)
#include "pat_dev.h"
#include "pat_ops.h"

namespace pat {

namespace {

typedef int v8i_t __attribute__((ext_vector_type(8)));

// Scale of a block whose largest finite element is amax: biased exponent of the smallest power of two with amax <= 448 2^e.
// amax = f 2^x with f in [1, 2): 448 = 1.75 * 2^8.  A block of zeros gets 2^0.
__device__ __forceinline__ int scale_code(float amax)
{
    if (amax == 0.f) return 127;
    int x;
    const float f = frexpf(amax, &x);                          // [0.5, 1): exact for subnormal numbers too
    const int e = x - (f <= 0.875f ? 9 : 8);
    return max(e, -127) + 127;
}
// x 2^-e, exactly: 2^(127 - code) is a normal number for every code but 254, which no fp32 element asks for (448 2^e stays below 2^128: e <= 119)
__device__ __forceinline__ float scaled(float x, int code) { return x * __uint_as_float((uint32_t)(254 - code) << 23); }

__device__ __forceinline__ float finite_abs(float x) { const float a = fabsf(x); return a < INFINITY ? a : 0.f; }     // NaN and infinity count as nothing

// sixteen elements as 8-bit values; what is not finite becomes the format's NaN
__device__ __forceinline__ uint4 to_f8(const float (&x)[16], int code)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(x[4 * i], code), scaled(x[4 * i + 1], code), 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled(x[4 * i + 2], code), scaled(x[4 * i + 3], code), v, true);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!(fabsf(x[4 * i + j]) < INFINITY)) w[i] |= 0x7Fu << (8 * j);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float one(const float *p) { return *p; }
__device__ __forceinline__ float one(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void sixteen(const float *p, float (&x)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 v = reinterpret_cast<const float4 *>(p)[i];
        x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
    }
}
__device__ __forceinline__ void sixteen(const uint16_t *p, float (&x)[16])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[8 * i + 2 * j] = bf16lo(w[j]); x[8 * i + 2 * j + 1] = bf16hi(w[j]); }
    }
}
// columns c .. c + 15 of a row (NULL: a row of padding), zeros behind column k
template <typename E>
__device__ __forceinline__ void load16(const E *row, int c, int k, bool vec, float (&x)[16])
{
    if (row && vec && c + 16 <= k) { sixteen(row + c, x); return; }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = row && c + i < k ? one(row + c + i) : 0.f;
}
__device__ __forceinline__ float amax16(const float (&x)[16])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, finite_abs(x[i]));
    return m;
}

// Activations: eight lanes hold a row's block; a workgroup two blocks of 16 rows.  Scales [KB4][16 tiles][4]: a word holds four
// blocks of one row, which is how the products' lanes load them.
template <typename E>
__global__ __launch_bounds__(256) void f8_pack_act_kernel(const E *x, int64_t ld, int m, int k, int KB, bool vec, uint4 *packed, uint8_t *scales, int Mp)
{
    const int r = threadIdx.x >> 3 & 15, piece = threadIdx.x & 7, kb = blockIdx.x * 2 + (threadIdx.x >> 7), tile = blockIdx.y, row = tile * 16 + r;
    if (kb >= KB) return;
    float v[16];
    load16(row < m ? x + (int64_t)row * ld : nullptr, kb * 128 + piece * 16, k, vec, v);
    float a = amax16(v);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) a = fmaxf(a, __shfl_xor(a, o, 64));
    const int code = scale_code(a);
    packed[((int64_t)tile * KB + kb) * 128 + (piece >> 2) * 64 + (piece & 3) * 16 + r] = to_f8(v, code);
    if (piece == 0) scales[((int64_t)(kb >> 2) * Mp + row) * 4 + (kb & 3)] = (uint8_t)code;
}

// Weights: a workgroup per block of 128 x 128, twice over the source: its largest element, then the values.  Scales [n / 128][KB4][4].
template <typename E>
__global__ __launch_bounds__(256) void f8_pack_weight_kernel(const E *w, int64_t ld, int n, int k, int KB, bool vec, uint4 *packed, uint8_t *scales, int KB4)
{
    __shared__ float top[4];
    const int kb = blockIdx.x, nb = blockIdx.y, piece = threadIdx.x & 7;
    float v[4][16], a = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = nb * 128 + i * 32 + (threadIdx.x >> 3);
        load16(row < n ? w + (int64_t)row * ld : nullptr, kb * 128 + piece * 16, k, vec, v[i]);
        a = fmaxf(a, amax16(v[i]));
    }
    a = wave_max(a);
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = a;
    __syncthreads();
    const int code = scale_code(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = nb * 128 + i * 32 + (threadIdx.x >> 3), tile = row >> 4;
        if (tile < (n + 15) / 16) packed[((int64_t)tile * KB + kb) * 128 + (piece >> 2) * 64 + (piece & 3) * 16 + (row & 15)] = to_f8(v[i], code);
    }
    if (threadIdx.x == 0) scales[((int64_t)nb * KB4 + (kb >> 2)) * 4 + (kb & 3)] = (uint8_t)code;
}

__device__ __forceinline__ v8i_t both(uint4 a, uint4 b) { return v8i_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w}; }

template <int S>
__device__ __forceinline__ floatx4_t mfma_f8(v8i_t a, v8i_t b, floatx4_t c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, S, sa, S, sb);
}

// eight 8-bit values as bf16, exactly
__device__ __forceinline__ bf16x8_t widen8(int lo, int hi)
{
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// a block's product by the bf16 instructions, scaled and added: |sum| 2^(both exponents) as a product of powers of two is exact
__device__ __forceinline__ floatx4_t mfma_wide(v8i_t a, v8i_t b, floatx4_t c, int sa, int sb)
{
    floatx4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a[2 * i], a[2 * i + 1]), widen8(b[2 * i], b[2 * i + 1]), s, 0, 0, 0);
    const int e = (sa & 255) + (sb & 255) - 254;
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] += __builtin_ldexpf(s[j], e);
    return c;
}

__device__ __forceinline__ void put(float *p, float v, bool add) { *p = add ? *p + v : v; }
__device__ __forceinline__ void put(uint16_t *p, float v, bool add) { *p = f32_to_bf16(add ? bf16_to_f32(*p) + v : v); }
__device__ __forceinline__ void put4(float *p, floatx4_t v, bool add)
{
    float4 o = make_float4(v[0], v[1], v[2], v[3]);
    if (add) { const float4 y = *reinterpret_cast<float4 *>(p); o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w; }
    *reinterpret_cast<float4 *>(p) = o;
}
__device__ __forceinline__ void put4(uint16_t *p, floatx4_t v, bool add)
{
    if (add) {
        const uint2 y = *reinterpret_cast<uint2 *>(p);
        v[0] += bf16lo(y.x); v[1] += bf16hi(y.x); v[2] += bf16lo(y.y); v[3] += bf16hi(y.y);
    }
    *reinterpret_cast<uint2 *>(p) = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16), (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
}
// rows n0 .. n0 + 3 of a tile's result for batch row m
template <typename E>
__device__ __forceinline__ void emit(const F8Args &a, int m, int n0, floatx4_t v)
{
    if (m >= a.m || n0 >= a.n) return;
    E *p = reinterpret_cast<E *>(a.y) + (int64_t)m * a.ldy + n0;
    if (a.vec && n0 + 4 <= a.n) { put4(p, v, a.add); return; }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (n0 + j < a.n) put(p + j, v[j], a.add);
}

// A wave takes one tile of 16 weight rows and four of the batch.
template <typename E>
__global__ __launch_bounds__(256) void f8_gemm_kernel(F8Args a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, KB = a.KB, KB4 = (KB + 3) / 4;
    const int nt = blockIdx.x * 4 + wave, m0 = blockIdx.y * 4, NT = (a.n + 15) / 16, MT = a.Mp / 16;
    if (nt >= NT) return;
    const uint4 *w = a.w + (int64_t)nt * KB * 128 + lane;
    const uint32_t *ws = a.ws + (int64_t)(nt >> 3) * KB4;
    floatx4_t acc[4] = {};
    for (int kb = 0; kb < KB; ++kb) {
        const v8i_t wf = both(w[kb * 128], w[kb * 128 + 64]);
        const int sw = ws[kb >> 2] >> (8 * (kb & 3));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int mt = min(m0 + t, MT - 1);
            const uint4 *x = a.x + ((int64_t)mt * KB + kb) * 128 + lane;
            const int sx = a.xs[(int64_t)(kb >> 2) * a.Mp + mt * 16 + (lane & 15)] >> (8 * (kb & 3));
            acc[t] = sizeof(E) == 4 ? mfma_wide(wf, both(x[0], x[64]), acc[t], sw, sx) : mfma_f8<0>(wf, both(x[0], x[64]), acc[t], sw, sx);
        }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) emit<E>(a, (m0 + t) * 16 + (lane & 15), nt * 16 + (lane >> 4) * 4, acc[t]);
}

}  // namespace

hipError_t launch_f8_pack_act(const void *x, bool f32, int64_t ld, int m, int k, void *packed, void *scales, hipStream_t s)
{
    const int KB = (k + 127) / 128, tiles = (m + 15) / 16, el = f32 ? 4 : 2;
    const bool vec = ((uintptr_t)x & 15) == 0 && ld * el % 16 == 0;
    const dim3 grid((unsigned)((KB + 1) / 2), (unsigned)tiles);
    if (f32) f8_pack_act_kernel<float><<<grid, 256, 0, s>>>((const float *)x, ld, m, k, KB, vec, (uint4 *)packed, (uint8_t *)scales, tiles * 16);
    else f8_pack_act_kernel<uint16_t><<<grid, 256, 0, s>>>((const uint16_t *)x, ld, m, k, KB, vec, (uint4 *)packed, (uint8_t *)scales, tiles * 16);
    return hipGetLastError();
}

hipError_t launch_f8_pack_weight(const void *w, bool f32, int64_t ld, int n, int k, void *packed, void *scales, hipStream_t s)
{
    const int KB = (k + 127) / 128, el = f32 ? 4 : 2;
    const bool vec = ((uintptr_t)w & 15) == 0 && ld * el % 16 == 0;
    const dim3 grid((unsigned)KB, (unsigned)((n + 127) / 128));
    if (f32) f8_pack_weight_kernel<float><<<grid, 256, 0, s>>>((const float *)w, ld, n, k, KB, vec, (uint4 *)packed, (uint8_t *)scales, (KB + 3) / 4);
    else f8_pack_weight_kernel<uint16_t><<<grid, 256, 0, s>>>((const uint16_t *)w, ld, n, k, KB, vec, (uint4 *)packed, (uint8_t *)scales, (KB + 3) / 4);
    return hipGetLastError();
}

hipError_t launch_f8_gemm(const F8Args &a, bool f32, hipStream_t s)
{
    const dim3 grid((unsigned)((a.n + 63) / 64), (unsigned)((a.Mp + 63) / 64));
    if (f32) f8_gemm_kernel<float><<<grid, 256, 0, s>>>(a);
    else f8_gemm_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace pat
