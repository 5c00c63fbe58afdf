// Host-side launchers of the operators of include/pat_operators.h (internal to libpat_decode.so).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pat {

// ---- rotation and append (kv_append.hip) ---------------------------------------
struct AppendArgs {
    const void *qkv;           // [rows, ld]: hq q heads, hkv k heads, hkv v heads
    void *q_out;               // [rows, ldq], the same type
    int64_t ld, ldq;
    uint16_t *k, *v;           // [n_pages][hkv][P][d] bf16
    const int32_t *seq, *pos, *page_table;
    const float *cs;           // [n_pos][d/2][cos, sin]
    const uint16_t *gq, *gk;   // [d] or NULL
    int32_t *skipped;          // NULL, or counts rows that name no place of the cache
    int rows, hq, hkv, n_pages, lgP, n_seqs, max_pages, n_pos;
    float eps;
};
hipError_t launch_kv_append(const AppendArgs &a, int d, bool f32, hipStream_t s);
hipError_t launch_rope_table(float *cs, int64_t n_pos, int d, double base, hipStream_t s);

// ---- decode attention of sequences that share prefixes (attn_shared.hip) ---------
constexpr int kSharedMaxSeqs = 2048;       // sequences (and groups) of a plan: the planning workgroup keeps them in LDS
constexpr int kSharedRows = 32;            // query rows (sequence, head of the KV head's group) of a record
// How much room a plan has: a part is one sequence's share of a record (a row block on a chunk of keys).
inline __host__ __device__ int64_t shared_parts(int n_seqs) { return 7 * (int64_t)n_seqs + 1024; }
inline __host__ __device__ int64_t shared_records(int n_seqs, int G) { return shared_parts(n_seqs) * ((G + kSharedRows - 1) / kSharedRows); }
struct SharedRecord {
    int32_t seq0;              // sequence of row 0
    int32_t r0, rows;          // rows r0 .. r0 + rows - 1: row r is head r % G of sequence seq0 + r / G
    int32_t table_row;         // whose pages hold the keys
    int32_t t0, cnt;           // keys t0 .. t0 + cnt - 1
    int32_t part0;             // part of sequence seq0
    int32_t pad;
};
struct SharedSeq {
    int32_t p0, p_step, pn;    // parts of the shared prefix
    int32_t s0, sn;            // parts of its own keys
    int32_t bad;               // its length or its group makes no sense
    int32_t pad[2];
};
struct SharedHeader {
    int32_t n_prefix, n_own;   // records of shared prefixes, then of sequences' own keys
    int32_t solo;              // own records: a wave takes a head by itself, four heads a workgroup
    int32_t prefix_chunk, own_chunk;
    int32_t mark, n_seqs, G, hkv;      // what the plan was made for: a call with anything else gives no numbers
    int32_t pad[7];
};
constexpr int32_t kSharedMark = 0x50415453;
inline int64_t shared_plan_bytes(int n_seqs, int G)
{
    // at least a SharedSeq for as many sequences as any plan has: a call made with a plan for fewer reads its own, and finds out, inside the buffer
    const int64_t used = n_seqs * (int64_t)sizeof(SharedSeq) + shared_records(n_seqs, G) * (int64_t)sizeof(SharedRecord), least = kSharedMaxSeqs * (int64_t)sizeof(SharedSeq);
    return (int64_t)sizeof(SharedHeader) + (used > least ? used : least);
}
struct SharedPlanArgs {
    const int32_t *kv_len, *group_start, *shared_len;
    int n_seqs, n_groups, max_len, hkv, G, n_cu;
    void *plan;
};
hipError_t launch_attn_plan(const SharedPlanArgs &a, hipStream_t s);
struct SharedArgs {
    const void *q;             // [n_seqs, ldq]
    void *out;                 // [n_seqs, ldo], the same type
    int64_t ldq, ldo;
    const uint16_t *k, *v;     // [n_pages][hkv][P][d] bf16
    const int32_t *page_table;
    const void *plan;
    float *part_acc, *part_ml; // [part][hq][d], [part][hq][max, sum]
    int n_seqs, hq, hkv, n_pages, lgP, max_pages;
};
hipError_t launch_attn_shared(const SharedArgs &a, int d, bool f32, int n_cu, hipStream_t s);

// ---- 8-bit projections (gemm_f8.hip) ---------------------------------------------
inline int64_t f8_operand_bytes(int64_t rows, int64_t k) { return (rows + 15) / 16 * ((k + 127) / 128) * 2048; }
inline int64_t f8_act_bytes(int64_t m, int64_t k) { return (m + 15) / 16 * ((k + 511) / 512) * 8192; }
inline int64_t f8_weight_scale_bytes(int64_t n, int64_t k) { return (n + 127) / 128 * ((k + 511) / 512) * 4; }
inline int64_t f8_act_scale_bytes(int64_t m, int64_t k) { return (m + 15) / 16 * 16 * ((k + 511) / 512) * 4; }
struct F8Args {
    const uint4 *w, *x;        // operands in tiles
    const uint32_t *ws, *xs;   // four scales a word: [n / 128][KB4], [KB4][Mp]
    void *y;                   // [m, ldy] fp32 or bf16
    int64_t ldy;
    int n, m, Mp, KB;          // Mp: m up to a multiple of 16; KB: blocks of 128 columns
    bool add, vec;             // y += ; rows n .. n + 3 of y by one store
    float *part;               // sums of K slices [slice][Mp][16-row tiles of n][16], where f8_tile has more than one
};
// Every workgroup of a product of few rows reads x whole.  Up to 64 KiB of it the product's waves bring it to 8 bits themselves (one row of 12288 x 4096: 12.2 us, 13.5
// with a launch before it); above, what that costs each workgroup passes the launch (16 rows of 12288 x 4096 13.5 and 13.4 us, of 4096 x 22016 31.5 and 22.4).
inline bool f8_takes_raw(int m, int k, bool x32) { return m <= 16 && (int64_t)m * k * (x32 ? 4 : 2) <= 65536; }
int f8_stream_tiles(int n, int MB, bool wide);        // up to 64 rows: tiles of weight rows per workgroup, for MB tiles of batch rows
struct F8Tile { int TN, W, slices; };      // above 64 rows: tiles of weight rows per workgroup, waves of 32 batch rows, cuts of K
F8Tile f8_tile(int n, int m, int KB, bool wide);      // wide: fp32 results
inline int64_t f8_part_bytes(int n, int m, int k)
{
    if (m <= 64) return 0;
    const int a = f8_tile(n, m, (k + 127) / 128, false).slices, b = f8_tile(n, m, (k + 127) / 128, true).slices, most = a > b ? a : b;
    return most > 1 ? (int64_t)most * ((m + 15) / 16 * 16) * ((n + 15) / 16 * 16) * 4 : 0;
}
hipError_t launch_f8_pack_act(const void *x, bool f32, int64_t ld, int m, int k, void *packed, void *scales, hipStream_t s);
hipError_t launch_f8_pack_weight(const void *w, bool f32, int64_t ld, int n, int k, void *packed, void *scales, hipStream_t s);
hipError_t launch_f8_gemm(const F8Args &a, bool f32, hipStream_t s);
// up to 16 rows, x as it is, brought to its 8-bit form by the product's own waves (F8Args::x, xs unused)
hipError_t launch_f8_gemm_raw(const F8Args &a, const void *x, bool x32, int64_t ldx, int k, bool y32, hipStream_t s);

}  // namespace pat
