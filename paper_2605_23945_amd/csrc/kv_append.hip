// Rotation of new tokens' queries and keys, and their keys' and values' way into the paged cache, as one launch.
//
// A row is one token of one sequence: the q, k and v heads that a projection left, fp32 or bf16.  Per q and k head, after
// an RMSNorm over its d features where the model has one (x g / sqrt(mean x^2 + eps)), features (j, j + d/2) turn by the angle
// that the table holds for the row's position:  a' = a cos - b sin,  b' = a sin + b cos,  in fp32.  q goes out in the
// input's type, k and v are rounded once, to the cache's bf16.
//
// What bounds it: memory.  A lane takes 16 bytes of a head's first half and the 16 bytes of their partners, so that a head is
// 4 to 16 lanes, every access is 16 bytes wide (8 where fp32 becomes the cache's bf16), and the norm's sum is a few lane exchanges.
// 10967 rows of 60 bf16 heads of 128 with the norm (338 MB read and written): 63 us, 5.3 TB/s, where a large copy reaches 5.0.  256 rows of 96 fp32
// heads: 5.0 us, one row of 24: 2.5 us, which are a launch and one chain of dependent reads (sequence, page, data).
#include "pat_dev.h"
#include "pat_ops.h"

namespace pat {

namespace {

struct F32 { typedef float4 vec; static constexpr int V = 4; };
struct Bf16 { typedef uint4 vec; static constexpr int V = 8; };

__device__ __forceinline__ void widen(float4 v, float *o) { o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w; }
__device__ __forceinline__ void widen(uint4 v, float *o)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { o[2 * i] = bf16lo(w[i]); o[2 * i + 1] = bf16hi(w[i]); }
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) { return (uint32_t)f32_to_bf16(a) | ((uint32_t)f32_to_bf16(b) << 16); }
__device__ __forceinline__ void store_bf16(uint16_t *p, const float (&v)[4]) { *reinterpret_cast<uint2 *>(p) = make_uint2(two_bf16(v[0], v[1]), two_bf16(v[2], v[3])); }
__device__ __forceinline__ void store_bf16(uint16_t *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store_same(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_same(uint16_t *p, const float (&v)[8]) { store_bf16(p, v); }

template <int D, typename T, typename E>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a)
{
    constexpr int V = T::V, LPH = D / 2 / V;                   // elements per access, lanes per head
    const uint32_t unit = blockIdx.x * (256 / LPH) + threadIdx.x / LPH;
    const int j = (threadIdx.x % LPH) * V, heads = a.hq + 2 * a.hkv;
    const uint32_t row = unit / (uint32_t)heads;
    const int head = (int)(unit - row * (uint32_t)heads);
    if (row >= (uint32_t)a.rows) return;                       // whole heads of lanes leave: the sums below stay within a head
    const int seq = a.seq[row], pos = a.pos[row];
    if (seq < 0) return;                                       // a row of padding
    bool ok = seq < a.n_seqs && pos >= 0 && pos < a.n_pos && (pos >> a.lgP) < a.max_pages;
    const int page = ok ? a.page_table[(int64_t)seq * a.max_pages + (pos >> a.lgP)] : -1;
    ok = ok && page >= 0 && page < a.n_pages;
    if (!ok) {
        if (a.skipped && head == 0 && j == 0) atomicAdd(a.skipped, 1);
        return;
    }
    const E *src = reinterpret_cast<const E *>(a.qkv) + (int64_t)row * a.ld + (int64_t)head * D;
    float x[V], y[V];
    widen(*reinterpret_cast<const typename T::vec *>(src + j), x);
    widen(*reinterpret_cast<const typename T::vec *>(src + j + D / 2), y);
    if (head < a.hq + a.hkv) {
        float4 cs[V / 2];
        const float4 *tab = reinterpret_cast<const float4 *>(a.cs + ((int64_t)pos * (D / 2) + j) * 2);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) cs[i] = tab[i];
        const uint16_t *g = head < a.hq ? a.gq : a.gk;
        if (g) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
            for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
            const float inv = 1.0f / sqrtf(ss / (float)D + a.eps);
#pragma unroll
            for (int i = 0; i < V; ++i) { x[i] = x[i] * inv * bf16_to_f32(g[j + i]); y[i] = y[i] * inv * bf16_to_f32(g[j + i + D / 2]); }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float c = i & 1 ? cs[i / 2].z : cs[i / 2].x, s = i & 1 ? cs[i / 2].w : cs[i / 2].y;
            const float u = x[i] * c - y[i] * s;
            y[i] = x[i] * s + y[i] * c;
            x[i] = u;
        }
    }
    if (head < a.hq) {
        E *dst = reinterpret_cast<E *>(a.q_out) + (int64_t)row * a.ldq + (int64_t)head * D;
        store_same(dst + j, x);
        store_same(dst + j + D / 2, y);
        return;
    }
    const int h = head - a.hq, isv = h >= a.hkv;
    uint16_t *dst = (isv ? a.v : a.k) + (((int64_t)page * a.hkv + (isv ? h - a.hkv : h)) * ((int64_t)1 << a.lgP) + (pos & ((1 << a.lgP) - 1))) * D;
    store_bf16(dst + j, x);
    store_bf16(dst + j + D / 2, y);
}

// cos and sin of pos * base^(-2 j / d), formed in 64 bits and rounded once: an fp32 angle of a far position is off by far more than the result's last bit
__global__ __launch_bounds__(256) void rope_table_kernel(float2 *cs, int64_t n, int half, double base)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int j = (int)(i % half);
    double s, c;
    sincos((double)(i / half) * pow(base, -(double)j / (double)half), &s, &c);
    cs[i] = make_float2((float)c, (float)s);
}

template <int D>
hipError_t launch_append(const AppendArgs &a, bool f32, hipStream_t s)
{
    const int lph = D / 2 / (f32 ? F32::V : Bf16::V);
    const int64_t units = (int64_t)a.rows * (a.hq + 2 * a.hkv), per = 256 / lph;
    const unsigned grid = (unsigned)((units + per - 1) / per);
    if (f32) kv_append_kernel<D, F32, float><<<grid, 256, 0, s>>>(a);
    else kv_append_kernel<D, Bf16, uint16_t><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs &a, int d, bool f32, hipStream_t s) { return d == 128 ? launch_append<128>(a, f32, s) : launch_append<64>(a, f32, s); }

hipError_t launch_rope_table(float *cs, int64_t n_pos, int d, double base, hipStream_t s)
{
    const int64_t n = n_pos * (d / 2);
    rope_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(reinterpret_cast<float2 *>(cs), n, d / 2, base);
    return hipGetLastError();
}

}  // namespace pat
