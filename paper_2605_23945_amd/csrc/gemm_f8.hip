// Projections with weights and activations in 8-bit floating point (4 exponent and 3 mantissa bits) and a power-of-two scale per
// block of 128:  x = 2^e q,  e the smallest integer with max|x| <= 448 2^e over the block (448 is the format's largest value), q
// rounded to nearest even.  Weights have a scale per 128 rows and 128 columns, activations one per row and 128 columns.
//   y[m, n] = sum over blocks b of 2^(ex[m, b] + ew[n / 128, b]) sum over k in b of qx[m, k] qw[n, k]
// The matrix instruction of 16 x 16 x 128 8-bit operands takes both exponents per operand row and multiplies them in, so a block is one
// instruction with nothing beside it, and sums stay in its fp32 accumulators.  It does not keep all bits of a block's smaller products
// (5e-6 of the result's norm on values of a normal distribution, 5e-5 on values of every exponent): nothing beside a bf16 result's own 2^-8, and it
// serves those.  For fp32 results the 8-bit values are widened to bf16 (exactly) and multiplied by the bf16 instructions, whose sums are fp32
// throughout, at half the rate; a block's sum is then scaled and added.
//
// Layout of both operands, [rows, k]: tiles of 16 rows, per tile and block of 128 columns 2 KiB: piece (half, g, r) of 16 bytes
// holds row r, columns half * 64 + g * 16 ..; lane g * 16 + r of a wave loads the pieces of both halves, 1 KiB per instruction.
// (The instruction would have 32 consecutive columns in a lane; any order does that both operands share.)
//
// What bounds it: the weights' bytes for few rows.  One row of 12288 x 4096 (50 MB): 9.9 us, 5.1 TB/s, launch and ramp included, of 6.0 that plain reads reach.  Where x
// comes packed and for many rows, the loads that the compiler's waits leave under way (see both kernels): 27 fp32 rows of 5120 x 6912 take 12 us, and 3 before it for x, where
// the bytes take 6; 251 rows of 22016 x 4096 30 and 4, where weights and products take 15 to 17 each; 5003 rows of 7168 x 8192 245 us and 19 for x, together 2.2 PFLOP/s
// (a library product of 8192 cubed 2.8, of these sizes 1.8).
#include "pat_dev.h"
#include "pat_ops.h"

namespace pat {

namespace {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef short shortx2_t __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
constexpr uint32_t kInfBits = 0x7F800000u;

// Scale of a block whose largest finite element is amax: biased exponent of the smallest power of two with amax <= 448 2^e.
// amax = f 2^x with f in [1, 2): 448 = 1.75 * 2^8.  A block of zeros gets 2^0.
__device__ __forceinline__ int scale_code(uint32_t top)
{
    const float amax = __uint_as_float(top);
    if (amax == 0.f) return 127;
    int x;
    const float f = frexpf(amax, &x);                          // [0.5, 1): exact for subnormal numbers too
    const int e = x - (f <= 0.875f ? 9 : 8);
    return max(e, -127) + 127;
}
// Sixteen consecutive elements of a row, as they lie in memory.
template <typename E> struct Piece;
template <> struct Piece<float> {
    uint32_t w[16];
    __device__ __forceinline__ void load(const float *p)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
    __device__ __forceinline__ void set(int i, const float *p) { w[i] = p ? __float_as_uint(*p) : 0u; }
    // the largest magnitude's bits; not below those of infinity if something is not finite
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
    __device__ __forceinline__ uint32_t top_finite() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, (w[i] & 0x7FFFFFFFu) < 0x7F800000u ? w[i] & 0x7FFFFFFFu : 0u);
        return m;
    }
    __device__ __forceinline__ bool finite(int i) const { return (w[i] & 0x7FFFFFFFu) < 0x7F800000u; }
    __device__ __forceinline__ uint4 to_f8(float scale) const
    {
        uint4 o;
        uint32_t *q = &o.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            shortx2_t v = {0, 0};
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, __uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 1]), scale, false);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, __uint_as_float(w[4 * i + 2]), __uint_as_float(w[4 * i + 3]), scale, true);
            q[i] = __builtin_bit_cast(uint32_t, v);
        }
        return o;
    }
};
template <> struct Piece<uint16_t> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const uint16_t *p)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
    __device__ __forceinline__ void set(int i, const uint16_t *p)
    {
        const uint32_t v = p ? *p : 0u;
        w[i >> 1] = i & 1 ? w[i >> 1] | v << 16 : v;
    }
    __device__ __forceinline__ uint32_t top() const
    {
        ushortx2_t m = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushortx2_t, w[i] & 0x7FFF7FFFu));
        return (uint32_t)max(m[0], m[1]) << 16;
    }
    __device__ __forceinline__ uint32_t top_finite() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, finite(i) ? (w[i >> 1] >> (i & 1 ? 16 : 0)) & 0x7FFFu : 0u);
        return m << 16;
    }
    __device__ __forceinline__ bool finite(int i) const { return ((w[i >> 1] >> (i & 1 ? 16 : 0)) & 0x7FFFu) < 0x7F80u; }
    __device__ __forceinline__ uint4 to_f8(float scale) const
    {
        uint4 o;
        uint32_t *q = &o.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            shortx2_t v = {0, 0};
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2_t, w[2 * i]), scale, false);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2_t, w[2 * i + 1]), scale, true);
            q[i] = __builtin_bit_cast(uint32_t, v);
        }
        return o;
    }
};
// columns c .. c + 15 of a row (NULL: a row of padding), zeros behind column k
template <typename E>
__device__ __forceinline__ void load16(const E *row, int c, int k, bool vec, Piece<E> &x)
{
    if (row && vec && c + 16 <= k) { x.load(row + c); return; }
#pragma unroll
    for (int i = 0; i < 16; ++i) x.set(i, row && c + i < k ? row + c + i : nullptr);
}
// x 2^-e rounded to the format by the conversion instruction, which divides by the scale's power of two; what is not finite becomes the format's NaN
template <typename E>
__device__ __forceinline__ uint4 to_f8(const Piece<E> &x, int code, bool all_finite)
{
    uint4 o = x.to_f8(__uint_as_float((uint32_t)code << 23));
    if (!all_finite) {
        uint32_t *q = &o.x;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!x.finite(i)) q[i >> 2] |= 0x7Fu << (8 * (i & 3));
    }
    return o;
}

// Activations: eight lanes hold a row's block; a workgroup two blocks of 16 rows.  Scales [KB4][16 tiles][4]: a word holds four
// blocks of one row, which is how the products' lanes load them; blocks are padded to that with zeros.  5003 rows of 8192 bf16: 19 us, 6.5 TB/s.
template <typename E>
__global__ __launch_bounds__(256) void f8_pack_act_kernel(const E *x, int64_t ld, int m, int k, int KB4, bool vec, uint4 *packed, uint8_t *scales, int Mp)
{
    const int r = threadIdx.x >> 3 & 15, piece = threadIdx.x & 7, kb = blockIdx.x * 2 + (threadIdx.x >> 7), tile = blockIdx.y, row = tile * 16 + r;
    Piece<E> v;
    load16(row < m ? x + (int64_t)row * ld : nullptr, kb * 128 + piece * 16, k, vec, v);
    uint32_t a = v.top();
    const bool fin = !__any(a >= kInfBits);
    if (!fin) a = v.top_finite();
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
    const int code = scale_code(a);
    packed[((int64_t)tile * KB4 * 4 + kb) * 128 + (piece >> 2) * 64 + (piece & 3) * 16 + r] = to_f8(v, code, fin);
    if (piece == 0) scales[((int64_t)(kb >> 2) * Mp + row) * 4 + (kb & 3)] = (uint8_t)code;
}

// Weights, once per program: a workgroup per block of 128 x 128, its elements in registers from the search for the largest to their rounding.  Scales
// [n / 128][KB4][4].  12288 x 4096 bf16: 33 us, 4.6 TB/s.
template <typename E>
__global__ __launch_bounds__(256) void f8_pack_weight_kernel(const E *w, int64_t ld, int n, int k, int KB, bool vec, uint4 *packed, uint8_t *scales, int KB4)
{
    __shared__ uint32_t top[4];
    const int kb = blockIdx.x, nb = blockIdx.y, piece = threadIdx.x & 7;
    Piece<E> v[4];
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = nb * 128 + i * 32 + (threadIdx.x >> 3);
        load16(row < n ? w + (int64_t)row * ld : nullptr, kb * 128 + piece * 16, k, vec, v[i]);
        a = max(a, v[i].top());
    }
    const bool fin = !__any(a >= kInfBits);
    if (!fin) a = max(max(v[0].top_finite(), v[1].top_finite()), max(v[2].top_finite(), v[3].top_finite()));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = a;
    __syncthreads();
    const int code = scale_code(max(max(top[0], top[1]), max(top[2], top[3])));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = nb * 128 + i * 32 + (threadIdx.x >> 3), tile = row >> 4;
        if (tile < (n + 15) / 16) packed[((int64_t)tile * KB + kb) * 128 + (piece >> 2) * 64 + (piece & 3) * 16 + (row & 15)] = to_f8(v[i], code, fin);
    }
    // the rest of a row's last word is 2^0: the products' padding multiplies by it, and a byte left as it was could be the scale that is no number
    if (threadIdx.x == 0)
        for (int i = kb; i < (kb == KB - 1 ? KB4 * 4 : kb + 1); ++i) scales[(int64_t)nb * KB4 * 4 + i] = (uint8_t)(i == kb ? code : 127);
}

__device__ __forceinline__ v8i_t both(uint4 a, uint4 b) { return v8i_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w}; }

template <int S>
__device__ __forceinline__ floatx4_t mfma_f8(v8i_t a, v8i_t b, floatx4_t c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, S, sa, S, sb);
}

// eight 8-bit values as bf16, exactly, times a power of two
__device__ __forceinline__ bf16x8_t widen8(int lo, int hi, float scale = 1.0f)
{
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
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
// A workgroup holds TN tiles of 16 weight rows; its eight waves take the blocks of columns in turn (wave w: w, w + 8, ...) and their
// sums meet in LDS, added in wave order.  A wave has registers for three blocks' operands (two above 32 rows): a block's weights and its part of x are
// requested together, two blocks (one) before they are multiplied.  Not all of that stays under way: packed x's scales are shifted right behind their request, for which
// the compiler waits for everything but the newest block's weights, and where the paths around the last blocks meet it waits for all of them, once in three (two) blocks.  Where x is small (RAW) every wave brings it to its 8-bit form
// itself, in the registers the product reads it from: lanes r, r + 16, r + 32 and r + 48 hold row r's block; no launch, no scratch and no barrier
// precede the stream.  Elsewhere x comes packed.
constexpr int kStreamWaves = 8;

__device__ __forceinline__ v8i_t both(u32x4_t a, u32x4_t b) { return v8i_t{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]}; }

template <int MB, int TN, bool RAW, typename X, typename E>
__global__ __launch_bounds__(kStreamWaves * 64) void f8_stream_kernel(F8Args a, const X *xraw, int64_t ldx, int k, bool xvec)
{
    __shared__ floatx4_t red[kStreamWaves][MB * TN][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int KB = a.KB, KB4 = (KB + 3) / 4, nt0 = blockIdx.x * TN, NT = (a.n + 15) / 16;
    const u32x4_t *w[TN];
    const uint32_t *ws[TN];
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        const int nt = min(nt0 + t, NT - 1);
        w[t] = reinterpret_cast<const u32x4_t *>(a.w) + (int64_t)nt * KB * 128 + lane;
        ws[t] = a.ws + (int64_t)(nt >> 3) * KB4;
    }
    const X *row = xraw + (int64_t)min(col, a.m - 1) * ldx;
    struct Packed { u32x4_t f[MB][2]; int s[MB]; };
    struct Raw { Piece<X> lo, hi; };
    struct Block { u32x4_t f[TN][2]; typename std::conditional<RAW, Raw, Packed>::type x; };
    auto load = [&](Block &b, int kb) {
        if (kb >= KB) return;
        if constexpr (RAW) {
            const int c = kb * 128 + g * 16;
            if (xvec && (kb + 1) * 128 <= k) { b.x.lo.load(row + c); b.x.hi.load(row + c + 64); }
            else { load16(row, c, k, false, b.x.lo); load16(row, c + 64, k, false, b.x.hi); }
        } else {
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const u32x4_t *x = reinterpret_cast<const u32x4_t *>(a.x) + ((int64_t)i * KB4 * 4 + kb) * 128 + lane;
                b.x.f[i][0] = x[0]; b.x.f[i][1] = x[64];
                b.x.s[i] = a.xs[(int64_t)(kb >> 2) * a.Mp + i * 16 + col] >> (8 * (kb & 3));
            }
        }
#pragma unroll
        for (int t = 0; t < TN; ++t) { b.f[t][0] = __builtin_nontemporal_load(w[t] + kb * 128); b.f[t][1] = __builtin_nontemporal_load(w[t] + kb * 128 + 64); }
    };
    floatx4_t acc[MB][TN] = {};
    auto multiply = [&](const Block &b, int kb) {
        if (kb >= KB) return;
        int sw[TN];
#pragma unroll
        for (int t = 0; t < TN; ++t) sw[t] = ws[t][kb >> 2] >> (8 * (kb & 3));
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            v8i_t xv;
            int sx;
            if constexpr (RAW) {                               // columns behind the batch repeat its last row; their results are dropped
                uint32_t top = max(b.x.lo.top(), b.x.hi.top());
                const bool fin = !__any(top >= kInfBits);
                if (!fin) top = max(b.x.lo.top_finite(), b.x.hi.top_finite());
                top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
                top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
                sx = scale_code(top);
                xv = both(to_f8(b.x.lo, sx, fin), to_f8(b.x.hi, sx, fin));
            } else {
                xv = both(b.x.f[i][0], b.x.f[i][1]);
                sx = b.x.s[i];
            }
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const v8i_t wv = both(b.f[t][0], b.f[t][1]);
                acc[i][t] = sizeof(E) == 4 ? mfma_wide(wv, xv, acc[i][t], sw[t], sx) : mfma_f8<0>(wv, xv, acc[i][t], sw[t], sx);
            }
        }
    };
    constexpr int W = kStreamWaves, R = MB > 2 ? 2 : 3;        // blocks in registers: with more of x, one on its way
    Block b[R];
#pragma unroll
    for (int i = 0; i < R - 1; ++i) load(b[i], wave + i * W);
    for (int kb = wave; kb < KB; kb += R * W)
#pragma unroll
        for (int i = 0; i < R; ++i) {
            load(b[(i + R - 1) % R], kb + (i + R - 1) * W);
            multiply(b[i], kb + i * W);
        }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t) red[wave][i * TN + t][lane] = acc[i][t];
    __syncthreads();
    for (int x = wave; x < MB * TN; x += W) {
        floatx4_t v = red[0][x][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            const floatx4_t u = red[i][x][lane];
            v[0] += u[0]; v[1] += u[1]; v[2] += u[2]; v[3] += u[3];
        }
        emit<E>(a, x / TN * 16 + col, (nt0 + x % TN) * 16 + g * 4, v);
    }
}

// ---- many rows: tiles on the matrix cores ------------------------------------------------------------------------------
// A workgroup of W waves holds TN tiles of 16 weight rows and 2 W tiles of 16 batch rows, a wave all TN and two of the batch's: weights go through LDS
// (asynchronous loads, S stages of TN x 2 KiB), where the waves share them; the batch's tiles are one wave's alone and go straight to
// registers, requested three blocks of columns ahead (x has just been written, so it comes from beyond the XCD's own L2).  Towards the end
// of a block all waves meet: the next block's weights have arrived, and the stage just read is requested anew.  Loads arrive in order,
// so a wave waits for its weights by the number of loads that it has issued since.  The compiler's wait for the next block's x counts its own loads alone, not those to LDS,
// and so leaves 8 loads under way (12 where scales were requested), whatever S: x is ahead by about one block and the weights by less.  For fp32 results it also brings the
// weights' scales to a scalar register where they are requested, once in four blocks, and waits for all loads but two there.
// The loop takes four blocks a turn, which one word of scales covers; K is padded to that with blocks of x that are zero.  There is no branch
// in it: the compiler moves matrix products past one.
constexpr int kBatchTiles = 2;      // four, on 512 registers, 276 us where two take 261 (5003 x 7168 x 8192, x's launch included)
template <int TN, int W, int S, typename E>
__global__ __launch_bounds__(W * 64, 2) void f8_tile_kernel(F8Args a, int nblk, int mblk, int slices)
{
    constexpr int TM = kBatchTiles, kStage = TN * 2048, NJ = 2 * TN / W;      // load instructions of a wave per stage
    constexpr int kAhead = 3;                                  // weight tiles in registers on their way from LDS: one tile's products are shorter than its read
    constexpr bool WIDE = sizeof(E) == 4;
    constexpr bool kTwo = 8 % TN != 0;                         // a workgroup's weight tiles may be of two blocks of 128 rows: two words of scales
    constexpr int kScales = TM + 1 + kTwo;                     // load instructions of load_scales
    __shared__ __align__(16) char lds[S * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int KB4 = (a.KB + 3) / 4, NT = (a.n + 15) / 16, MT = a.Mp / 16;
    // workgroups of an XCD (index mod 8) take neighbouring tiles: four columns of batch blocks, then the next weights
    int nb, mb, sl;
    {
        const int T = nblk * mblk * slices, xcd = blockIdx.x & 7, q = T >> 3, r = T & 7;
        int L = xcd * q + min(xcd, r) + (blockIdx.x >> 3);
        sl = L / (nblk * mblk);
        L -= sl * nblk * mblk;
        const int band = L / (nblk * 4), w = min(4, mblk - band * 4), i = L - band * nblk * 4;
        nb = i / w; mb = band * 4 + i - nb * w;
    }
    const int first = sl * KB4 / slices * 4, end = (sl + 1) * KB4 / slices * 4;       // this workgroup's blocks of columns
    const uint32_t lds0 = lds_offset(lds);
    const char *wsrc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int idx = wave * NJ + j;                         // half idx % 2 of weight tile idx / 2
        wsrc[j] = reinterpret_cast<const char *>(a.w) + (int64_t)min(nb * TN + (idx >> 1), NT - 1) * a.KB * 2048 + (idx & 1) * 1024;
    }
    auto fetch = [&](int kb, int slot) {
        const int64_t at = (int64_t)min(kb, a.KB - 1) * 2048;
#pragma unroll
        for (int j = 0; j < NJ; ++j) load_to_lds(wsrc[j] + at, lane * 16, lds0 + slot * kStage + (wave * NJ + j) * 1024);
    };
    const u32x4_t *xsrc[TM];
    const uint32_t *xss[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int mt = min((mb * W + wave) * TM + i, MT - 1);
        xsrc[i] = reinterpret_cast<const u32x4_t *>(a.x) + (int64_t)mt * KB4 * 512 + lane;
        xss[i] = a.xs + mt * 16 + col;
    }
    const uint32_t *wss = a.ws + (int64_t)(nb * TN >> 3) * KB4, *wss2 = a.ws + (int64_t)min((nb * TN + TN - 1) >> 3, (NT - 1) >> 3) * KB4;
    const int edge = 8 - (nb * TN & 7);                        // weight tiles from here on are of the next 128 rows
    struct Batch { u32x4_t lo[TM], hi[TM]; };
    struct Scales { uint32_t x[TM], w, w2; };
    auto load_batch = [&](Batch &b, int kb) {
        const int at = min(kb, KB4 * 4 - 1) * 128;
#pragma unroll
        for (int i = 0; i < TM; ++i) { b.lo[i] = xsrc[i][at]; b.hi[i] = xsrc[i][at + 64]; }
    };
    auto load_scales = [&](Scales &c, int kb) {
        const int at = min(kb >> 2, KB4 - 1);
#pragma unroll
        for (int i = 0; i < TM; ++i) c.x[i] = xss[i][(int64_t)at * a.Mp];
        c.w = wss[at];
        if constexpr (kTwo) c.w2 = wss2[at];
    };
    auto pin = [&](Batch &b) {                                 // here, or the compiler waits for newer loads than it needs to later
#pragma unroll
        for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(b.lo[i]), "+v"(b.hi[i]));
    };
    auto weight = [&](int slot, int t, u32x4_t (&f)[2]) {
        const char *p = lds + slot * kStage + t * 2048 + lane * 16;
        f[0] = *reinterpret_cast<const u32x4_t *>(p); f[1] = *reinterpret_cast<const u32x4_t *>(p + 1024);
    };
    floatx4_t acc[TN][TM] = {};
    Batch b[4];
    Scales c, cn;
    u32x4_t wf[4][2];
#pragma unroll
    for (int i = 0; i < S; ++i) fetch(first + i, i);
    load_scales(c, first);
#pragma unroll
    for (int i = 0; i < 3; ++i) load_batch(b[i], first + i);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int t = 0; t < kAhead; ++t) weight(0, t, wf[t]);
    int slot = 0;
    for (int kb = first; kb < end; kb += 4) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u == 0) load_scales(cn, kb + 4);
            load_batch(b[(u + 3) & 3], kb + u + 3);
            const int sw = c.w >> (8 * u), sw2 = kTwo ? (int)(c.w2 >> (8 * u)) : sw;
            // fp32 results: x widened once for all weight tiles (they are of one block of 128 rows), and the factor 2^(both exponents) of the block's sums: what of
            // it an fp32 number does not hold goes into the widened x, whose sums are then beyond the result's range in any case
            bf16x8_t xw[WIDE ? TM : 1][4];
            float by[WIDE ? TM : 1];
            if constexpr (WIDE) {
                static_assert(!kTwo, "a workgroup's weight tiles have one scale");
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int e = (int)(c.x[i] >> (8 * u) & 255) + (sw & 255) - 254, r = min(max(e, -126), 127), rest = max(e - r, -126);
                    const float f = __uint_as_float((uint32_t)(rest + 127) << 23);
                    const v8i_t xv = both(b[u].lo[i], b[u].hi[i]);
                    by[i] = __uint_as_float((uint32_t)(r + 127) << 23);
#pragma unroll
                    for (int j = 0; j < 4; ++j) xw[i][j] = widen8(xv[2 * j], xv[2 * j + 1], f);
                }
            }
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                // or all of the block's weights are read ahead, into registers that the sums need; fp32 results' four tiles leave room, and their chains of four
                // products per tile go on side by side (100 x 12288 x 4096: 28.7 us with the fence, 26.3 without)
                if constexpr (!WIDE) __builtin_amdgcn_sched_barrier(0);
                if (t + kAhead == TN) {
                    // newer than the next block's weights: x of S - 1 blocks, weights of S - 2, and the scales where they were among them.
                    // One too many would let a wave read weights that have not arrived; this wait alone holds them back.
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"((S - 1) * 2 * TM + (S - 2) * NJ + (u < S - 1 ? kScales : 0)) : "memory");
                    pin(b[(u + 1) & 3]);
                    asm volatile("s_barrier" ::: "memory");
                    fetch(kb + u + S, slot);
                    slot = slot + 1 == S ? 0 : slot + 1;
                }
                if (t + kAhead < TN) weight(slot, t + kAhead, wf[(t + kAhead) & 3]);
                else weight(slot, t + kAhead - TN, wf[(t + kAhead) & 3]);
                const v8i_t wv = both(wf[t & 3][0], wf[t & 3][1]);
                const int s = !kTwo || t < edge ? sw : sw2;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    if constexpr (WIDE) {
                        floatx4_t p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < 4; ++j) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(wv[2 * j], wv[2 * j + 1]), xw[i][j], p, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[t][i][j] = fmaf(p[j], by[i], acc[t][i][j]);
                    } else {
                        acc[t][i] = mfma_f8<0>(wv, both(b[u].lo[i], b[u].hi[i]), acc[t][i], s, (int)(c.x[i] >> (8 * u)));
                    }
                }
            }
        }
        c = cn;
    }
    static_assert(TN % 4 == 0 && (S - 1) * 2 * TM + (S - 2) * NJ + kScales <= 63, "the next block's first weights land where this step's begin; the counter has six bits");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // nothing may arrive in LDS that has gone to another workgroup
    if (slices > 1) {                                          // fp32 sums of the slice: [slice][batch row][weight row]
        float *part = a.part + (int64_t)sl * a.Mp * NT * 16;
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int mt = (mb * W + wave) * TM + i, nt = nb * TN + t;
                if (mt < MT && nt < NT) *reinterpret_cast<floatx4_t *>(part + ((int64_t)(mt * 16 + col) * NT + nt) * 16 + g * 4) = acc[t][i];
            }
        return;
    }
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            emit<E>(a, ((mb * W + wave) * TM + i) * 16 + col, (nb * TN + t) * 16 + g * 4, acc[t][i]);
        }
}

// the slices' sums, added in their order
template <typename E>
__global__ __launch_bounds__(256) void f8_join_kernel(F8Args a, int slices)
{
    const int NT = (a.n + 15) / 16;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.m * NT * 4;
    if (i >= per) return;
    const int m = (int)(i / (NT * 4)), n4 = (int)(i - (int64_t)m * NT * 4);
    const floatx4_t *p = reinterpret_cast<const floatx4_t *>(a.part) + i;
    floatx4_t v = p[0];
    for (int s = 1; s < slices; ++s) {
        const floatx4_t u = p[(int64_t)s * a.Mp * NT * 4];
        v[0] += u[0]; v[1] += u[1]; v[2] += u[2]; v[3] += u[3];
    }
    emit<E>(a, m, n4 * 4, v);
}

template <int TN, int W, int S, typename E>
hipError_t launch_tile(const F8Args &a, int slices, hipStream_t s)
{
    const int NT = (a.n + 15) / 16, nblk = (NT + TN - 1) / TN, mblk = (a.m + W * 32 - 1) / (W * 32);
    f8_tile_kernel<TN, W, S, E><<<(unsigned)(nblk * mblk * slices), W * 64, 0, s>>>(a, nblk, mblk, slices);
    if (slices > 1) f8_join_kernel<E><<<(unsigned)(((int64_t)a.m * NT * 4 + 255) / 256), 256, 0, s>>>(a, slices);
    return hipGetLastError();
}

// Tiles of a workgroup: as few as leave one workgroup per compute unit, up to three.  27 fp32 rows of 5120 x 6912 by 1, 2 and 3 tiles, x's launch included: 19.8, 17.3
// and 19.0 us; of 22016 x 4096: 29.7, 28.5 and 25.8; one row of 12288 x 4096: 14.3, 15.4 and 12.2.  fp32 results of four batch tiles leave no registers for three
// (60 rows of 12288 x 4096: 30 us, 24 by two).
constexpr int stream_most(int MB, bool wide) { return MB == 4 && wide ? 2 : 3; }

template <int MB, bool RAW, typename X, typename E>
hipError_t launch_stream(const F8Args &a, const X *x, int64_t ldx, int k, bool vec, hipStream_t s)
{
    constexpr int kMost = stream_most(MB, sizeof(E) == 4);
    const int NT = (a.n + 15) / 16, TN = f8_stream_tiles(a.n, MB, sizeof(E) == 4);
    if (TN == 1) f8_stream_kernel<MB, 1, RAW, X, E><<<NT, kStreamWaves * 64, 0, s>>>(a, x, ldx, k, vec);
    else if (TN == 2) f8_stream_kernel<MB, 2, RAW, X, E><<<(NT + 1) / 2, kStreamWaves * 64, 0, s>>>(a, x, ldx, k, vec);
    else f8_stream_kernel<MB, kMost, RAW, X, E><<<(NT + kMost - 1) / kMost, kStreamWaves * 64, 0, s>>>(a, x, ldx, k, vec);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_product(const F8Args &a, hipStream_t s)
{
    const int MT = a.Mp / 16;
    if (MT <= 4) {
        switch (MT) {
        case 1: return launch_stream<1, false, float, E>(a, nullptr, 0, 0, false, s);
        case 2: return launch_stream<2, false, float, E>(a, nullptr, 0, 0, false, s);
        case 3: return launch_stream<3, false, float, E>(a, nullptr, 0, 0, false, s);
        default: return launch_stream<4, false, float, E>(a, nullptr, 0, 0, false, s);
        }
    }
    const F8Tile t = f8_tile(a.n, a.m, a.KB, sizeof(E) == 4);
    if constexpr (sizeof(E) == 4) return launch_tile<4, 4, 4, E>(a, t.slices, s);
    else if (t.W == 8) return t.TN == 12 ? launch_tile<12, 8, 4, E>(a, t.slices, s) : launch_tile<8, 8, 4, E>(a, t.slices, s);
    else return t.TN == 12 ? launch_tile<12, 4, 3, E>(a, t.slices, s) : t.TN == 8 ? launch_tile<8, 4, 4, E>(a, t.slices, s) : launch_tile<4, 4, 4, E>(a, t.slices, s);
}

}  // namespace

int f8_stream_tiles(int n, int MB, bool wide)
{
    const int NT = (n + 15) / 16, most = stream_most(MB, wide);
    return NT <= 256 ? 1 : NT <= 512 ? 2 : most;
}

// Weight tiles and waves of a workgroup and cuts of K.  A workgroup keeps a compute unit about as busy as two do, so the time is rounds of
// 256 workgroups, blocks of columns in each and a block's time: 0.36, 0.55 and 0.75 us for 4, 8 and 12 tiles by four waves, 1.0 and 1.37 us for 8 and 12 by eight
// (measured on products of 100 to 5003 rows), 0.7 us for fp32 results (0.63 measured: what a cut costs them is a little less than the rule says); a cut K costs a launch and its sums' way out and back.  Measured, x's launch included, 5003 x 7168 x 8192: 12 tiles by
// eight waves 274 us, by four 283, 8 tiles 288 and 294; 2048 x 8192 x 8192: 161, 146, 130 and 144; 251 x 22016 x 4096: 48, 38, 39 and 47; 128 x 22016 x 4096: 45, 37, 34 and 33,
// 4 tiles 35; 100 x 12288 x 4096: 41, 32, 30 and 28, 4 tiles 21; 251 x 4096 x 11008: two slices of 4 tiles 31, four of 8 31, one of 4 42.  The rule takes the best of each.
F8Tile f8_tile(int n, int m, int KB, bool wide)
{
    const int NT = (n + 15) / 16, KB4 = (KB + 3) / 4;
    F8Tile best{4, 4, 1};
    double least = 1e300;
    for (int w = 4; w <= (wide ? 4 : 8); w += 4)
        for (int tn = w; tn <= (wide ? 4 : 12); tn += 4)
            for (int sl = 1; sl <= 8 && sl <= KB4; ++sl) {     // a slice has a word of scales at least
                const int64_t wg = (int64_t)((NT + tn - 1) / tn) * ((m + 32 * w - 1) / (32 * w)) * sl;
                const double block = wide ? 0.7 : w == 4 ? 0.17 + 0.048 * tn : 0.22 + 0.096 * tn;
                const double cost = (double)((wg + 255) / 256) * ((KB4 + sl - 1) / sl * 4) * block + (sl > 1 ? 5.0 + (double)m * n * sl * 8 / 4e6 : 0.0);
                if (cost < least) { least = cost; best = F8Tile{tn, w, sl}; }
            }
    return best;
}

hipError_t launch_f8_pack_act(const void *x, bool f32, int64_t ld, int m, int k, void *packed, void *scales, hipStream_t s)
{
    const int KB4 = (k + 511) / 512, tiles = (m + 15) / 16, el = f32 ? 4 : 2;
    const bool vec = ((uintptr_t)x & 15) == 0 && ld * el % 16 == 0;
    const dim3 grid((unsigned)(KB4 * 2), (unsigned)tiles);
    if (f32) f8_pack_act_kernel<float><<<grid, 256, 0, s>>>((const float *)x, ld, m, k, KB4, vec, (uint4 *)packed, (uint8_t *)scales, tiles * 16);
    else f8_pack_act_kernel<uint16_t><<<grid, 256, 0, s>>>((const uint16_t *)x, ld, m, k, KB4, vec, (uint4 *)packed, (uint8_t *)scales, tiles * 16);
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

hipError_t launch_f8_gemm(const F8Args &a, bool f32, hipStream_t s) { return f32 ? launch_product<float>(a, s) : launch_product<uint16_t>(a, s); }

hipError_t launch_f8_gemm_raw(const F8Args &a, const void *x, bool x32, int64_t ldx, int k, bool y32, hipStream_t s)
{
    const bool vec = ((uintptr_t)x & 15) == 0 && ldx * (x32 ? 4 : 2) % 16 == 0;
    if (x32) return y32 ? launch_stream<1, true, float, float>(a, (const float *)x, ldx, k, vec, s) : launch_stream<1, true, float, uint16_t>(a, (const float *)x, ldx, k, vec, s);
    return y32 ? launch_stream<1, true, uint16_t, float>(a, (const uint16_t *)x, ldx, k, vec, s) : launch_stream<1, true, uint16_t, uint16_t>(a, (const uint16_t *)x, ldx, k, vec, s);
}

}  // namespace pat
