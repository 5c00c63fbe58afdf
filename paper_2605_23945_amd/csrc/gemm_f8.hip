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

// ---- few rows: weights streamed once, straight into registers ------------------------------------------------------
// A workgroup holds one tile of 16 weight rows; its eight waves take the blocks of columns in turn (wave w: w, w + 8, ...), four at a time, so
// that 8 KiB of weights are in flight per wave, and their sums meet in LDS, added in wave order.  Up to 16 rows (RAW) every wave
// brings x to its 8-bit form itself, in the registers the product reads it from: lanes r, r + 16, r + 32 and r + 48 hold row r's block, no launch, no
// scratch and no barrier precede the stream.  Above, x comes packed.
constexpr int kStreamWaves = 8, kStreamAhead = 4;

__device__ __forceinline__ uint4 load_once(const uint4 *p)
{
    const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
    return make_uint4(v[0], v[1], v[2], v[3]);
}

template <int MB, bool RAW, typename X, typename E>
__global__ __launch_bounds__(kStreamWaves * 64) void f8_stream_kernel(F8Args a, const X *xraw, int64_t ldx, int k, bool xvec)
{
    __shared__ floatx4_t red[kStreamWaves][MB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int KB = a.KB, KB4 = (KB + 3) / 4, nt = blockIdx.x;
    const uint4 *w = a.w + (int64_t)nt * KB * 128 + lane;
    const uint32_t *ws = a.ws + (int64_t)(nt >> 3) * KB4;
    floatx4_t acc[MB] = {};
    for (int k0 = wave; k0 < KB; k0 += kStreamWaves * kStreamAhead) {
        uint4 wf[kStreamAhead][2];
#pragma unroll
        for (int u = 0; u < kStreamAhead; ++u) {
            const int kb = min(k0 + u * kStreamWaves, KB - 1);
            wf[u][0] = load_once(w + kb * 128); wf[u][1] = load_once(w + kb * 128 + 64);
        }
#pragma unroll
        for (int u = 0; u < kStreamAhead; ++u) {
            const int kb = k0 + u * kStreamWaves;
            if (kb >= KB) break;
            const int sw = ws[kb >> 2] >> (8 * (kb & 3));
            const v8i_t wv = both(wf[u][0], wf[u][1]);
#pragma unroll
            for (int t = 0; t < MB; ++t) {
                v8i_t xv;
                int sx;
                if (RAW) {
                    float lo[16], hi[16];
                    const X *row = col < a.m ? xraw + (int64_t)col * ldx : nullptr;
                    load16(row, kb * 128 + g * 16, k, xvec, lo);
                    load16(row, kb * 128 + 64 + g * 16, k, xvec, hi);
                    float top = fmaxf(amax16(lo), amax16(hi));
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    sx = scale_code(top);
                    xv = both(to_f8(lo, sx), to_f8(hi, sx));
                } else {
                    const uint4 *x = a.x + ((int64_t)t * KB + kb) * 128 + lane;
                    xv = both(x[0], x[64]);
                    sx = a.xs[(int64_t)(kb >> 2) * a.Mp + t * 16 + col] >> (8 * (kb & 3));
                }
                acc[t] = sizeof(E) == 4 ? mfma_wide(wv, xv, acc[t], sw, sx) : mfma_f8<0>(wv, xv, acc[t], sw, sx);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < MB; ++t) red[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave < MB) {
        floatx4_t v = red[0][wave][lane];
#pragma unroll
        for (int i = 1; i < kStreamWaves; ++i) {
            const floatx4_t u = red[i][wave][lane];
            v[0] += u[0]; v[1] += u[1]; v[2] += u[2]; v[3] += u[3];
        }
        emit<E>(a, wave * 16 + col, nt * 16 + g * 4, v);
    }
}

// ---- many rows: tiles on the matrix cores ------------------------------------------------------------------------------
// A workgroup holds TN tiles of 16 weight rows and 4 TM tiles of 16 batch rows, a wave all TN and TM of the batch's: weights go through LDS
// (asynchronous loads, two stages of TN x 2 KiB), where the four waves share them; the batch's tiles are one wave's alone and go straight to
// registers, a block of columns ahead.  Before the last weight tile of a block all waves meet: what the next block needs has arrived, and
// the stage just read is requested anew.
template <int TN, int TM, typename E>
__global__ __launch_bounds__(256) void f8_tile_kernel(F8Args a, int nblk, int mblk)
{
    constexpr int kStage = TN * 2048, NJ = TN / 2;             // load instructions of a wave per stage
    constexpr bool WIDE = sizeof(E) == 4;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int KB = a.KB, KB4 = (KB + 3) / 4, NT = (a.n + 15) / 16, MT = a.Mp / 16;
    // workgroups of an XCD (index mod 8) take neighbouring tiles: four columns of batch blocks, then the next weights
    int nb, mb;
    {
        const int T = nblk * mblk, xcd = blockIdx.x & 7, q = T >> 3, r = T & 7;
        const int L = xcd * q + min(xcd, r) + (blockIdx.x >> 3);
        const int band = L / (nblk * 4), w = min(4, mblk - band * 4), i = L - band * nblk * 4;
        nb = i / w; mb = band * 4 + i - nb * w;
    }
    const uint32_t lds0 = lds_offset(lds);
    const char *wsrc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int idx = wave * NJ + j;
        wsrc[j] = reinterpret_cast<const char *>(a.w) + (int64_t)min(nb * TN + (idx >> 1), NT - 1) * KB * 2048 + (idx & 1) * 1024;
    }
    auto fetch = [&](int kb) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) load_to_lds(wsrc[j] + (int64_t)min(kb, KB - 1) * 2048, lane * 16, lds0 + (kb & 1) * kStage + (wave * NJ + j) * 1024);
    };
    const uint4 *xsrc[TM];
    const uint32_t *xss[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int mt = min((mb * 4 + wave) * TM + i, MT - 1);
        xsrc[i] = a.x + (int64_t)mt * KB * 128 + lane;
        xss[i] = a.xs + mt * 16 + col;
    }
    const uint32_t *wss = a.ws + (int64_t)(nb * TN >> 3) * KB4, *wss2 = a.ws + (int64_t)min((nb * TN + TN - 1) >> 3, (NT - 1) >> 3) * KB4;
    const int edge = 8 - (nb * TN & 7);                        // weight tiles from here on are of the next 128 rows
    struct Batch { u32x4_t lo[TM], hi[TM]; uint32_t s[TM], w, w2; };
    auto load_batch = [&](Batch &b, int kb) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            b.lo[i] = *reinterpret_cast<const u32x4_t *>(xsrc[i] + kb * 128); b.hi[i] = *reinterpret_cast<const u32x4_t *>(xsrc[i] + kb * 128 + 64);
            b.s[i] = xss[i][(int64_t)(kb >> 2) * a.Mp];
        }
        b.w = wss[kb >> 2]; b.w2 = wss2[kb >> 2];
    };
    auto pin = [&](Batch &b) {                                 // here, or the compiler waits for all loads at every later use
#pragma unroll
        for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(b.lo[i]), "+v"(b.hi[i]), "+v"(b.s[i]));
        asm volatile("" : "+v"(b.w), "+v"(b.w2));
    };
    auto weight = [&](int kb, int t, u32x4_t (&f)[2]) {
        const char *p = lds + (kb & 1) * kStage + t * 2048 + lane * 16;
        f[0] = *reinterpret_cast<const u32x4_t *>(p); f[1] = *reinterpret_cast<const u32x4_t *>(p + 1024);
    };
    floatx4_t acc[TN][TM] = {};
    Batch b0, b1;
    u32x4_t wf[2][2];
    fetch(0);
    load_batch(b0, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    pin(b0);
    asm volatile("s_barrier" ::: "memory");
    fetch(1);
    weight(0, 0, wf[0]);
    // No branch in here: the compiler moves matrix products past one.  Behind the last block the last one's operands are read again, for nothing.
    auto step = [&](int kb, Batch &b, Batch &next) {
        load_batch(next, min(kb + 1, KB - 1));
        const int sh = 8 * (kb & 3);
        const int sw = b.w >> sh, sw2 = b.w2 >> sh;
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            __builtin_amdgcn_sched_barrier(0);                 // or all of the block's weights are read ahead, into registers that the sums need
            if (t + 1 < TN) weight(kb, t + 1, wf[(t + 1) & 1]);
            else {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                pin(next);
                asm volatile("s_barrier" ::: "memory");
                fetch(kb + 2);
                weight(kb + 1, 0, wf[(t + 1) & 1]);
            }
            const u32x4_t f0 = wf[t & 1][0], f1 = wf[t & 1][1];
            const v8i_t wv = v8i_t{(int)f0[0], (int)f0[1], (int)f0[2], (int)f0[3], (int)f1[0], (int)f1[1], (int)f1[2], (int)f1[3]};
            const int s = t < edge ? sw : sw2;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const u32x4_t l = b.lo[i], h = b.hi[i];
                const v8i_t xv = v8i_t{(int)l[0], (int)l[1], (int)l[2], (int)l[3], (int)h[0], (int)h[1], (int)h[2], (int)h[3]};
                const int sx = b.s[i] >> sh;
                acc[t][i] = WIDE ? mfma_wide(wv, xv, acc[t][i], s, sx) : mfma_f8<0>(wv, xv, acc[t][i], s, sx);
            }
        }
    };
    static_assert(TN % 2 == 0, "the next block's first weights land where this step's begin");
    int kb = 0;
    for (; kb + 1 < KB; kb += 2) { step(kb, b0, b1); step(kb + 1, b1, b0); }
    if (kb < KB) step(kb, b0, b1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // nothing may arrive in LDS that has gone to another workgroup
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            emit<E>(a, ((mb * 4 + wave) * TM + i) * 16 + col, (nb * TN + t) * 16 + g * 4, acc[t][i]);
        }
}

template <int TN, int TM, typename E>
hipError_t launch_tile(const F8Args &a, hipStream_t s)
{
    const int nblk = ((a.n + 15) / 16 + TN - 1) / TN, mblk = (a.Mp / 16 + 4 * TM - 1) / (4 * TM);
    f8_tile_kernel<TN, TM, E><<<(unsigned)(nblk * mblk), 256, 2 * TN * 2048, s>>>(a, nblk, mblk);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_product(const F8Args &a, int n_cu, hipStream_t s)
{
    const int NT = (a.n + 15) / 16, MT = a.Mp / 16;
    if (MT <= 4) {
        switch (MT) {
        case 1: f8_stream_kernel<1, false, float, E><<<NT, kStreamWaves * 64, 0, s>>>(a, nullptr, 0, 0, false); break;
        case 2: f8_stream_kernel<2, false, float, E><<<NT, kStreamWaves * 64, 0, s>>>(a, nullptr, 0, 0, false); break;
        case 3: f8_stream_kernel<3, false, float, E><<<NT, kStreamWaves * 64, 0, s>>>(a, nullptr, 0, 0, false); break;
        default: f8_stream_kernel<4, false, float, E><<<NT, kStreamWaves * 64, 0, s>>>(a, nullptr, 0, 0, false); break;
        }
        return hipGetLastError();
    }
    if constexpr (sizeof(E) == 4) return MT <= 8 ? launch_tile<4, 2, E>(a, s) : launch_tile<4, 4, E>(a, s);
    else {
    if (MT <= 8) return launch_tile<8, 2, E>(a, s);
    // workgroups in rounds of the compute units: the height that ends the last round soonest
    const int mblk = (MT + 15) / 16;
    auto cost = [&](int tn, int per_cu) { const int64_t wg = (int64_t)((NT + tn - 1) / tn) * mblk, slots = (int64_t)n_cu * per_cu; return (wg + slots - 1) / slots * tn * per_cu; };
    const int64_t c6 = cost(6, 2), c8 = cost(8, 2), c12 = cost(12, 1), c16 = cost(16, 1);
    if (c16 <= c12 && c16 <= c8 && c16 <= c6) return launch_tile<16, 4, E>(a, s);
    if (c12 <= c8 && c12 <= c6) return launch_tile<12, 4, E>(a, s);
    return c8 <= c6 ? launch_tile<8, 4, E>(a, s) : launch_tile<6, 4, E>(a, s);
    }
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

hipError_t launch_f8_gemm(const F8Args &a, bool f32, int n_cu, hipStream_t s) { return f32 ? launch_product<float>(a, n_cu, s) : launch_product<uint16_t>(a, n_cu, s); }

hipError_t launch_f8_gemm_raw(const F8Args &a, const void *x, bool x32, int64_t ldx, int k, bool y32, hipStream_t s)
{
    const unsigned grid = (unsigned)((a.n + 15) / 16);
    const bool vec = ((uintptr_t)x & 15) == 0 && ldx * (x32 ? 4 : 2) % 16 == 0;
    if (x32) {
        if (y32) f8_stream_kernel<1, true, float, float><<<grid, kStreamWaves * 64, 0, s>>>(a, (const float *)x, ldx, k, vec);
        else f8_stream_kernel<1, true, float, uint16_t><<<grid, kStreamWaves * 64, 0, s>>>(a, (const float *)x, ldx, k, vec);
    } else {
        if (y32) f8_stream_kernel<1, true, uint16_t, float><<<grid, kStreamWaves * 64, 0, s>>>(a, (const uint16_t *)x, ldx, k, vec);
        else f8_stream_kernel<1, true, uint16_t, uint16_t><<<grid, kStreamWaves * 64, 0, s>>>(a, (const uint16_t *)x, ldx, k, vec);
    }
    return hipGetLastError();
}

}  // namespace pat
