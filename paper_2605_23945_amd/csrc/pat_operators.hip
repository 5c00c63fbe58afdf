// C entry points of include/pat_operators.h: what the host can check of the arguments, then the launch.  Nothing here throws or
// allocates, and everything is enqueued on the caller's stream, so the calls can be captured into a graph.
#include "../../include/pat_operators.h"
#include "pat_ops.h"
#include "row_overlap.h"

#include <atomic>

using namespace pat;

namespace {

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool type_ok(int t) { return t == PAT_F32 || t == PAT_BF16; }
int64_t size_of(int t) { return t == PAT_F32 ? 4 : 2; }
bool cache_ok(int32_t n_pages, int32_t page_tokens, int32_t d)
{
    return n_pages > 0 && (page_tokens == 16 || page_tokens == 32 || page_tokens == 64 || page_tokens == 128) && (d == 64 || d == 128);
}
int lg(int v) { return __builtin_ctz((unsigned)v); }
int done(hipError_t e) { return e == hipSuccess ? PAT_OK : PAT_EHIP; }

// compute units of the current device, looked up once per device
int compute_units()
{
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    n = known[dev].load(std::memory_order_relaxed);
    if (n) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
    known[dev].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace

extern "C" {

int pat_op_rope_table(int64_t n_pos, int32_t head_dim, double base, float *cos_sin, void *stream)
{
    if (!cos_sin || !aligned(cos_sin, 16) || n_pos <= 0 || n_pos > (1 << 25) || (head_dim != 64 && head_dim != 128) || !(base > 1.0)) return PAT_EINVAL;
    return done(launch_rope_table(cos_sin, n_pos, head_dim, base, (hipStream_t)stream));
}

int pat_op_kv_append(const void *qkv, int32_t type, int64_t ld, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                     const int32_t *seq, const int32_t *pos, const float *cos_sin, int32_t n_pos, const void *gq, const void *gk, float eps,
                     void *k_pages, void *v_pages, int32_t n_pages, int32_t page_tokens, const int32_t *page_table, int32_t n_seqs, int32_t max_pages,
                     void *q_out, int64_t ldq, int32_t *skipped, void *stream)
{
    if (rows < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads > 4096 || n_kv_heads > 4096 || !type_ok(type) || !cache_ok(n_pages, page_tokens, head_dim)) return PAT_EINVAL;
    const int64_t width = ((int64_t)n_q_heads + 2 * n_kv_heads) * head_dim, el = size_of(type);
    if (rows == 0) return PAT_OK;
    if (!qkv || !seq || !pos || !cos_sin || !k_pages || !v_pages || !page_table || !q_out || n_pos <= 0 || n_seqs <= 0 || max_pages <= 0) return PAT_EINVAL;
    if (ld < width || ldq < (int64_t)n_q_heads * head_dim || ld * el % 16 || ldq * el % 16) return PAT_EINVAL;
    if (!aligned(qkv, 16) || !aligned(q_out, 16) || !aligned(cos_sin, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16)) return PAT_EINVAL;
    if ((gq == nullptr) != (gk == nullptr) || !(eps >= 0.f) || rows * (width / head_dim) >= ((int64_t)1 << 28) - (type == PAT_F32 && head_dim == 128 ? 15 : 0))
        return PAT_EINVAL;                                     // up to 16 lanes a head, in workgroups of 256 below 2^32 of them
    const bool in_place = q_out == qkv && (ldq == ld || rows == 1);
    if (!in_place && rows_overlap(qkv, ld * el, width * el, q_out, ldq * el, (int64_t)n_q_heads * head_dim * el, rows)) return PAT_EINVAL;
    AppendArgs a{};
    a.qkv = qkv; a.q_out = q_out; a.ld = ld; a.ldq = ldq; a.k = (uint16_t *)k_pages; a.v = (uint16_t *)v_pages;
    a.seq = seq; a.pos = pos; a.page_table = page_table; a.cs = cos_sin; a.gq = (const uint16_t *)gq; a.gk = (const uint16_t *)gk; a.skipped = skipped;
    a.rows = rows; a.hq = n_q_heads; a.hkv = n_kv_heads; a.n_pages = n_pages; a.lgP = lg(page_tokens); a.n_seqs = n_seqs; a.max_pages = max_pages;
    a.n_pos = n_pos; a.eps = eps;
    return done(launch_kv_append(a, head_dim, type == PAT_F32, (hipStream_t)stream));
}

static bool heads_ok(int32_t n_seqs, int32_t hq, int32_t hkv)
{
    return n_seqs > 0 && n_seqs <= kSharedMaxSeqs && hq > 0 && hkv > 0 && hq % hkv == 0 && hq <= 4096;
}

int64_t pat_op_attn_plan_bytes(int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads)
{
    return heads_ok(n_seqs, n_q_heads, n_kv_heads) ? shared_plan_bytes(n_seqs, n_q_heads / n_kv_heads) : -1;
}

int64_t pat_op_attn_scratch_bytes(int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (!heads_ok(n_seqs, n_q_heads, n_kv_heads) || (head_dim != 64 && head_dim != 128)) return -1;
    return shared_parts(n_seqs) * n_q_heads * (head_dim + 2) * 4;
}

int pat_op_attn_plan(const int32_t *kv_len, const int32_t *group_start, const int32_t *shared_len, int32_t n_seqs, int32_t n_groups, int32_t max_len,
                     int32_t n_q_heads, int32_t n_kv_heads, void *plan, void *stream)
{
    if (!heads_ok(n_seqs, n_q_heads, n_kv_heads) || !kv_len || !group_start || !shared_len || !plan || !aligned(plan, 16)) return PAT_EINVAL;
    if (n_groups <= 0 || n_groups > kSharedMaxSeqs || max_len <= 0 || max_len > (1 << 30)) return PAT_EINVAL;
    SharedPlanArgs a{kv_len, group_start, shared_len, n_seqs, n_groups, max_len, n_kv_heads, n_q_heads / n_kv_heads, compute_units(), plan};
    return done(launch_attn_plan(a, (hipStream_t)stream));
}

int pat_op_attn_shared(const void *q, int32_t type, int64_t ldq, int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                       const void *k_pages, const void *v_pages, int32_t n_pages, int32_t page_tokens, const int32_t *page_table, int32_t max_pages,
                       const void *plan, void *out, int64_t ldo, void *scratch, void *stream)
{
    if (!heads_ok(n_seqs, n_q_heads, n_kv_heads) || !type_ok(type) || !cache_ok(n_pages, page_tokens, head_dim)) return PAT_EINVAL;
    const int64_t el = size_of(type), width = (int64_t)n_q_heads * head_dim;
    if (!q || !k_pages || !v_pages || !page_table || !plan || !out || !scratch || max_pages <= 0 || ldq < width || ldo < width || ldq * el % 16 || ldo * el % 16) return PAT_EINVAL;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(plan, 16) || !aligned(scratch, 256)) return PAT_EINVAL;
    SharedArgs a{};
    a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo; a.k = (const uint16_t *)k_pages; a.v = (const uint16_t *)v_pages; a.page_table = page_table; a.plan = plan;
    a.part_acc = (float *)scratch;
    a.part_ml = a.part_acc + shared_parts(n_seqs) * n_q_heads * head_dim;
    a.n_seqs = n_seqs; a.hq = n_q_heads; a.hkv = n_kv_heads; a.n_pages = n_pages; a.lgP = lg(page_tokens); a.max_pages = max_pages;
    return done(launch_attn_shared(a, head_dim, type == PAT_F32, compute_units(), (hipStream_t)stream));
}

static bool product_ok(int32_t n, int32_t k) { return n > 0 && k > 0 && n <= (1 << 22) && k <= (1 << 20); }

int64_t pat_op_f8_weight_bytes(int32_t n, int32_t k) { return product_ok(n, k) ? f8_operand_bytes(n, k) : -1; }
int64_t pat_op_f8_scale_bytes(int32_t n, int32_t k) { return product_ok(n, k) ? f8_weight_scale_bytes(n, k) : -1; }

int pat_op_f8_pack_weight(const void *w, int32_t type, int64_t ld, int32_t n, int32_t k, void *packed, void *scales, void *stream)
{
    if (!product_ok(n, k) || !type_ok(type) || !w || !packed || !scales || ld < k || !aligned(packed, 256) || !aligned(scales, 4) || !aligned(w, size_of(type))) return PAT_EINVAL;
    return done(launch_f8_pack_weight(w, type == PAT_F32, ld, n, k, packed, scales, (hipStream_t)stream));
}

static bool batch_ok(int32_t n, int32_t k, int32_t m) { return product_ok(n, k) && m >= 0 && m <= (1 << 19) && (int64_t)m * n <= ((int64_t)1 << 36); }

static int64_t part_offset(int32_t m, int32_t k) { return (f8_act_bytes(m, k) + f8_act_scale_bytes(m, k) + 255) / 256 * 256; }

int64_t pat_op_f8_gemm_scratch_bytes(int32_t n, int32_t k, int32_t m)
{
    return batch_ok(n, k, m) ? part_offset(m, k) + f8_part_bytes(n, m, k) : -1;
}

int pat_op_f8_gemm_plan(int32_t n, int32_t k, int32_t m, int32_t x_type, int32_t y_type, int32_t plan[5])
{
    if (!plan || !batch_ok(n, k, m) || m == 0 || !type_ok(x_type) || !type_ok(y_type)) return PAT_EINVAL;
    const bool wide = y_type == PAT_F32;
    if (m <= 64) {
        plan[0] = f8_takes_raw(m, k, x_type == PAT_F32) ? 0 : 1;
        plan[2] = (m + 15) / 16; plan[1] = f8_stream_tiles(n, plan[2], wide); plan[3] = 8; plan[4] = 1;
        return PAT_OK;
    }
    const F8Tile t = f8_tile(n, m, (k + 127) / 128, wide);
    plan[0] = 2; plan[1] = t.TN; plan[2] = 2 * t.W; plan[3] = t.W; plan[4] = t.slices;
    return PAT_OK;
}

int pat_op_f8_gemm(const void *w_packed, const void *w_scales, int32_t n, int32_t k, const void *x, int32_t x_type, int64_t ldx, int32_t m, void *y,
                   int32_t y_type, int64_t ldy, int32_t mode, void *scratch, void *stream)
{
    if (!batch_ok(n, k, m) || !type_ok(x_type) || !type_ok(y_type) || mode < 0 || mode > 1) return PAT_EINVAL;
    if (!w_packed || !w_scales || !aligned(w_packed, 256) || !aligned(w_scales, 4) || ldx < k || ldy < n) return PAT_EINVAL;
    if (m == 0) return PAT_OK;
    if (!x || !y || !scratch || !aligned(x, size_of(x_type)) || !aligned(y, size_of(y_type)) || !aligned(scratch, 256)) return PAT_EINVAL;
    if (rows_overlap(x, ldx * size_of(x_type), k * size_of(x_type), y, ldy * size_of(y_type), n * size_of(y_type), m)) return PAT_EINVAL;
    char *sc = (char *)scratch + f8_act_bytes(m, k);
    F8Args a{};
    a.w = (const uint4 *)w_packed; a.x = (const uint4 *)scratch; a.ws = (const uint32_t *)w_scales; a.xs = (const uint32_t *)sc;
    a.y = y; a.ldy = ldy; a.n = n; a.m = m; a.Mp = (m + 15) / 16 * 16; a.KB = (k + 127) / 128; a.add = mode == 1;
    a.part = (float *)((char *)scratch + part_offset(m, k));
    a.vec = aligned(y, 4 * size_of(y_type)) && ldy % 4 == 0;
    if (f8_takes_raw(m, k, x_type == PAT_F32)) return done(launch_f8_gemm_raw(a, x, x_type == PAT_F32, ldx, k, y_type == PAT_F32, (hipStream_t)stream));
    const hipError_t e = launch_f8_pack_act(x, x_type == PAT_F32, ldx, m, k, scratch, sc, (hipStream_t)stream);
    return e != hipSuccess ? PAT_EHIP : done(launch_f8_gemm(a, y_type == PAT_F32, (hipStream_t)stream));
}

}  // extern "C"
