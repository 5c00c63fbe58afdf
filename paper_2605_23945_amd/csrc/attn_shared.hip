// Decode attention of sequences that share prefixes, over the paged cache: one query token per sequence, several answers to
// one prompt in a group.  softmax(q K^T / sqrt(d)) V over a sequence's keys is a sum over any cut of them: each piece gives
// its maximum, its sum and its weighted values, and pieces are joined by exp(m_i - m) (fp32 throughout).  So a group's shared
// keys are one piece for all its sequences: their query heads on a KV head are the rows of ONE matrix product with the shared
// K and V, which are read once, and each sequence's own keys are pieces of their own.
//
// Planning (once per step, on the device, from the lengths there): records (rows, keys) of about equal work, see
// attn_plan_kernel.  A record is a block of up to 32 rows on a chunk of keys; per KV head it is one workgroup's item whose
// four waves take tiles of 32 keys in turn ("together"), or, for sequences' own keys on four and more KV heads, a wave takes a
// head by itself and a workgroup four heads.  A wave streams its own tiles: K and V by asynchronous loads to its 16 KiB of LDS (32 keys of
// 128 features), the K half requested anew as soon as its fragments are in registers, the V half likewise, so no wave waits
// for another while it streams.  Both products run on the matrix cores with a row per operand column:
//   S^T[key, row] = K q^T,   O^T[feature, row] += V^T p^T    (V read transposed from LDS)
// q is exact in one bf16 term where it is bf16 and in three where it is fp32; p to 2^-17 in two rounded terms beside bf16 outputs
// (whose own rounding is 2^-8), and exact in three beside fp32 ones.  K's and V's fragments serve two row tiles of a bf16 record;
// fp32 ones take their tiles in turn.
//
// What bounds it: K's and V's bytes where there are many.  256 sequences of 16 groups on 32 KV heads (1.98 GB): 325 us and 6.4 for the join, 6.1 TB/s, the
// rate of plain reads; 64 sequences on one prefix of 8190 keys and 20 KV heads (302 MB): 54 and 4.6 us.  Small ones are a chain of dependent steps: the record, q and
// the pages (1.5 us), the first K (3 us), its tiles, the waves' meeting, the join's launch; and a grid for all the records that a plan has room for, most of whose
// workgroups find none: three sequences of 50 keys 4.8 and 3.9 us.  128 on one KV head with fp32 queries (56 MB): 22 and 4, where a record of more than 16 rows walks its
// chain and its keys twice.  The plan takes 13 to 16 us, once for all of a step's layers.
#include "attn_mfma_dev.h"
#include "pat_ops.h"

namespace pat {

namespace {

constexpr int kTile = 32;       // keys per tile
constexpr int kW = 4;           // waves of a workgroup
constexpr int kPlan = 1024;     // threads of the planning workgroup

// ---- the plan --------------------------------------------------------------------------------------------------

__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t *tmp)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    int64_t t = 0;
    for (int i = 0; i < kPlan / 64; ++i) t += tmp[i];
    __syncthreads();
    return t;
}

// off[i] := sum of off[0 .. i - 1], off[n] := the sum; n <= 2 * kPlan, off holds n + 1 entries
__device__ void block_scan(int32_t *off, int n, int32_t *tmp)
{
    const int i = 2 * threadIdx.x, lane = threadIdx.x & 63;
    const int a = i < n ? off[i] : 0, b = i + 1 < n ? off[i + 1] : 0;
    int v = a + b;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    if (lane == 63) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) base += tmp[w];
    const int end = base + v;
    if (i < n) off[i] = end - a - b;
    if (i + 1 < n) off[i + 1] = end - b;
    if ((i == n - 1) || (i + 1 == n - 1)) off[n] = end;
    __syncthreads();
}

// the last i of [0, n) with off[i] <= x
__device__ __forceinline__ int find(const int32_t *off, int n, int x)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (off[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// how many records on, at n workgroups each dealt to eight XCDs in turn, a workgroup of the same XCD comes
__device__ __forceinline__ int xcd_stride(int n) { return (n & 7) == 0 ? 1 : 8 / (n & -n); }

__device__ __forceinline__ int up(int64_t v, int to) { return (int)((v + to - 1) / to * to); }

// One workgroup.  A group shares its prefix if at least two of its sequences reach its end; others, and sequences shorter
// than their group's prefix, are read whole through their own rows.  Chunks: an item costs about two and a half tiles of 32 keys
// per wave beside its own, and two workgroups are resident on a compute unit; of 1 to 8 tiles per wave the number is taken that makes rounds times an item's
// cost least, with half a chunk for every row block's last one, and never one so short that the parts pass what shared_parts() holds.
__global__ __launch_bounds__(kPlan) void attn_plan_kernel(SharedPlanArgs a)
{
    __shared__ int32_t gcnt[kSharedMaxSeqs], gfirst[kSharedMaxSeqs], grec[kSharedMaxSeqs + 1], gpart[kSharedMaxSeqs + 1], srec[kSharedMaxSeqs + 1];
    __shared__ int64_t tmp[kPlan / 64];
    __shared__ int32_t wrong;
    const int tid = threadIdx.x, n = a.n_seqs, ng = a.n_groups, G = a.G, GB = (G + kSharedRows - 1) / kSharedRows;
    SharedHeader *head = reinterpret_cast<SharedHeader *>(a.plan);
    SharedSeq *seqs = reinterpret_cast<SharedSeq *>(head + 1);
    SharedRecord *recs = reinterpret_cast<SharedRecord *>(seqs + n);
    if (tid == 0) wrong = 0;
    for (int g = tid; g < ng; g += kPlan) { gcnt[g] = 0; gfirst[g] = n; }
    __syncthreads();
    for (int g = tid; g < ng; g += kPlan) {
        const int lo = a.group_start[g], hi = a.group_start[g + 1];
        if (lo < 0 || hi < lo || hi > n || (g == 0 && lo != 0) || (g == ng - 1 && hi != n)) wrong = 1;
    }
    __syncthreads();
    const bool bad_groups = wrong != 0;
    int len[2], grp[2];
    bool bad[2], in[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = tid + i * kPlan;
        len[i] = 0; grp[i] = 0; bad[i] = bad_groups; in[i] = false;
        if (s >= n || bad_groups) continue;
        const int L = a.kv_len[s];
        bad[i] = L < 0 || L > a.max_len;
        len[i] = bad[i] ? 0 : L;
        grp[i] = find(a.group_start, ng, s);
        const int S = a.shared_len[grp[i]];
        in[i] = S > 0 && len[i] >= S;
        if (in[i]) { atomicAdd(&gcnt[grp[i]], 1); atomicMin(&gfirst[grp[i]], s); }
    }
    __syncthreads();
    // work: row blocks times keys of the groups and of the sequences, and parts times keys
    int64_t wp = 0, ws = 0, pp = 0, nb = 0, ns = 0;            // and their row blocks
    int from[2];                                               // first key that sequence s reads by itself
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        in[i] = in[i] && gcnt[grp[i]] >= 2;
        from[i] = in[i] ? a.shared_len[grp[i]] : 0;
        ws += (int64_t)GB * (len[i] - from[i]);
        ns += len[i] > from[i] ? GB : 0;
    }
    for (int g = tid; g < ng; g += kPlan)
        if (gcnt[g] >= 2) {
            const int members = a.group_start[g + 1] - a.group_start[g];
            nb += (members * G + kSharedRows - 1) / kSharedRows;
            wp += (int64_t)((members * G + kSharedRows - 1) / kSharedRows) * a.shared_len[g];
            pp += (int64_t)members * a.shared_len[g];
        }
    wp = block_sum(wp, tmp); ws = block_sum(ws, tmp); pp = block_sum(pp, tmp); nb = block_sum(nb, tmp); ns = block_sum(ns, tmp);
    const bool solo = a.hkv % kW == 0;
    int c = 32;
    float least = INFINITY;
    for (int t = 1; t <= 8; ++t) {                             // tiles of a wave
        const float keys = (float)(32 * t), own = solo ? (float)ws / keys : (float)ws / (keys * kW);
        const float items = (float)a.hkv * ((float)wp / (keys * kW) + 0.5f * (float)nb) + (float)(solo ? a.hkv / kW : a.hkv) * (own + 0.5f * (float)ns);
        const float rounds = items / (float)(2 * a.n_cu), cost = (rounds <= 1.f ? 1.f : rounds + 0.3f) * (2.5f + (float)t);
        if (cost < least) { least = cost; c = 32 * t; }
    }
    const int64_t room = 2 * (int64_t)n + 512;                 // chunks beyond the first of each group's members, or sequence
    const int64_t most = 1 << 29;                              // a chunk's end stays an int; lengths are at most 2^30
    const int CP = max(c * kW, up(min(pp / room + 1, most), kTile * kW)), CS = max(solo ? c : c * kW, up(min(ws / room + 1, most), kTile));

    for (int g = tid; g < ng; g += kPlan) {
        const int members = bad_groups ? 0 : a.group_start[g + 1] - a.group_start[g];
        const int nc = gcnt[g] >= 2 ? (a.shared_len[g] + CP - 1) / CP : 0;
        grec[g] = nc * ((members * G + kSharedRows - 1) / kSharedRows);
        gpart[g] = nc * members;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = tid + i * kPlan;
        if (s < n) srec[s] = len[i] > from[i] ? (len[i] - (from[i] & ~15) + CS - 1) / CS : 0;
    }
    __syncthreads();
    int32_t *t32 = reinterpret_cast<int32_t *>(tmp);
    block_scan(grec, ng, t32); block_scan(gpart, ng, t32); block_scan(srec, n, t32);
    const int np = grec[ng], parts = gpart[ng], no = srec[n];
    if (tid == 0) {
        head->n_prefix = np; head->n_own = no * GB; head->solo = solo ? 1 : 0;
        head->prefix_chunk = CP; head->own_chunk = CS;
        head->mark = kSharedMark; head->n_seqs = n; head->G = G; head->hkv = a.hkv;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = tid + i * kPlan;
        if (s >= n) continue;
        SharedSeq q{};
        q.bad = bad[i] ? 1 : 0;
        if (in[i]) {
            const int g = grp[i], lo = a.group_start[g];
            q.p0 = gpart[g] + (s - lo); q.p_step = a.group_start[g + 1] - lo; q.pn = (a.shared_len[g] + CP - 1) / CP;
        }
        q.s0 = parts + srec[s]; q.sn = srec[s + 1] - srec[s];
        seqs[s] = q;
    }
    // A chunk's row blocks read the same keys: they come D records apart, so that their workgroups, hkv to a record and dealt to the eight XCDs in
    // turn, share an XCD's L2.
    const int D = xcd_stride(a.hkv);
    for (int r = tid; r < np; r += kPlan) {
        const int g = find(grec, ng, r), k = r - grec[g], lo = a.group_start[g], members = a.group_start[g + 1] - lo;
        const int nb = (members * G + kSharedRows - 1) / kSharedRows, nc = (a.shared_len[g] + CP - 1) / CP;
        const int blk = k / (D * nb), rem = k - blk * D * nb, w = min(D, nc - blk * D), rb = rem / w, ch = blk * D + rem - rb * w;
        SharedRecord e{};
        e.seq0 = lo; e.r0 = rb * kSharedRows; e.rows = min(kSharedRows, members * G - e.r0);
        e.table_row = gfirst[g];
        e.t0 = ch * CP; e.cnt = min(CP, a.shared_len[g] - e.t0);
        e.part0 = gpart[g] + ch * members;
        recs[r] = e;
    }
    for (int r = tid; r < no * GB; r += kPlan) {
        const int x = r / GB, s = find(srec, n, x), ch = x - srec[s];
        SharedRecord e{};
        const int L = a.kv_len[s], g = find(a.group_start, ng, s), S = a.shared_len[g];
        const int f = S > 0 && L >= S && gcnt[g] >= 2 ? S : 0, base = f & ~15;
        e.seq0 = s; e.r0 = (r - x * GB) * kSharedRows; e.rows = min(kSharedRows, G - e.r0);
        e.table_row = s;
        e.t0 = max(f, base + ch * CS); e.cnt = min(base + (ch + 1) * CS, L) - e.t0;
        e.part0 = parts + x;
        recs[np + r] = e;
    }
}

// ---- the pieces --------------------------------------------------------------------------------------------------

template <int N>
__device__ __forceinline__ void wait_newer() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }     // all but the N newest loads have arrived

// the largest of the four lanes of a column (lanes i, i + 16, i + 32, i + 48), in all of them: by exchanges between lane rows, without a way through LDS
__device__ __forceinline__ float column_max(float v)
{
    const uint32_t b = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const float m = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

__device__ __forceinline__ uint32_t two_bf16(float a, float b) { return (uint32_t)f32_to_bf16(a) | ((uint32_t)f32_to_bf16(b) << 16); }

template <bool F32> struct QTerms { static constexpr int n = F32 ? 3 : 1, p = F32 ? 3 : 2; };

// eight consecutive features of a query row as operand terms
__device__ __forceinline__ void load_q(const uint16_t *p, u32x4_t (&t)[1]) { t[0] = *reinterpret_cast<const u32x4_t *>(p); }
__device__ __forceinline__ void load_q(const float *p, u32x4_t (&t)[3])
{
    const float4 x = reinterpret_cast<const float4 *>(p)[0], y = reinterpret_cast<const float4 *>(p)[1];
    const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    split3_bf16(v, t[0], t[1], t[2]);
}

// p as two bf16 terms, each rounded to nearest: p - h - m is at most 2^-17 p, of either sign.  (Truncated terms, as many instructions and the same times, leave up to
// 2^-15 p and every result 1e-5 short in the mean: the sum that it is divided by is of whole p's.)
__device__ __forceinline__ void split2_bf16(const float *p, u32x4_t &h, u32x4_t &m)
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float x = p[2 * w], y = p[2 * w + 1];
        h[w] = two_bf16(x, y);
        m[w] = two_bf16(x - bf16lo(h[w]), y - bf16hi(h[w]));
    }
}

// RT row tiles of 16 on the tiles w0, w0 + ws, ... of a record's keys, one KV head; leaves its sums in o, M (scores in units of log2) and den.
template <int D, int RT, bool F32>
__device__ __forceinline__ bool stream_keys(const SharedArgs &a, const SharedRecord &e, int h, int w0, int ws, char *ring, bool once, floatx4_t (&o)[RT][D / 16],
                                            float (&M)[RT], float (&den)[RT])
{
    typedef typename std::conditional<F32, float, uint16_t>::type E;
    constexpr int KST = D / 32, FT = D / 16, PC = D / 8, KPI = 64 / PC, NI = kTile / KPI, kHalf = kTile * D * 2;
    constexpr int QT = QTerms<F32>::n, PT = QTerms<F32>::p;
    const int lane = threadIdx.x & 63, col = lane & 15, g4 = lane >> 4;
    const int G = a.hq / a.hkv, lgP = a.lgP, P = 1 << lgP;
    const int last = e.t0 + e.cnt - 1, tb = e.t0 & ~15, tiles = (last - tb) / kTile + 1;
    const bool beyond = (last >> lgP) >= a.max_pages;          // keys that no page holds: nothing of the record is read, its rows are no number
    const int n = tiles > w0 && !beyond ? (tiles - w0 + ws - 1) / ws : 0;
    const int64_t page_bytes = (int64_t)(a.hkv << lgP) * D * 2, head_bytes = (int64_t)(h << lgP) * D * 2;
    const char *kpool = reinterpret_cast<const char *>(a.k) + head_bytes, *vpool = reinterpret_cast<const char *>(a.v) + head_bytes;
    const uint32_t to = lds_offset(ring);
    bool bad = beyond;
    int page = 0;
    // lane i holds the page of half i % 2 (16 keys lie in one page) of the wave's tile (i / 2) of the next 32
    auto look_up = [&](int i0) {
        const int j = min(tb + ((i0 + (lane >> 1)) * ws + w0) * kTile + (lane & 1) * 16, last) >> lgP;
        page = a.page_table[(int64_t)e.table_row * a.max_pages + min(j, a.max_pages - 1)];
        asm volatile("" : "+v"(page));                         // here, or the compiler waits for all loads at every later use
        const bool wrong = j >= a.max_pages || page < 0 || page >= a.n_pages;
        if (wrong) page = 0;
        bad |= __any(wrong) != 0;
    };
    // Where the halves of the wave's tile i lie in both pools, and the lane's place in them: 16 keys of a page are consecutive, so inside the
    // record's keys a load's address is a sum of one scalar and one of NI / 2 constants.
    uint32_t place[NI / 2];
#pragma unroll
    for (int u = 0; u < NI / 2; ++u) {
        const int key = u * KPI + lane / PC;
        place[u] = (uint32_t)(key * (D * 2) + ((lane % PC) ^ (key & (PC - 1))) * 16);
    }
    struct Halves { int64_t at[2]; bool inside; int key0; };
    auto halves = [&](int i) {
        Halves t;
        t.key0 = tb + (i * ws + w0) * kTile;
        t.inside = t.key0 >= e.t0 && t.key0 + kTile - 1 <= last;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            t.at[j] = __builtin_amdgcn_readlane(page, 2 * (i & 31) + j) * page_bytes + (int64_t)((t.inside ? (t.key0 + j * 16) & (P - 1) : 0) * (D * 2));
        return t;
    };
    auto request = [&](const char *pool, const Halves &t, uint32_t at) {
        if (t.inside && once) {
#pragma unroll
            for (int u = 0; u < NI; ++u) load_to_lds_stream(pool + t.at[u / (NI / 2)], place[u % (NI / 2)], at + u * 1024);
        } else if (t.inside) {
#pragma unroll
            for (int u = 0; u < NI; ++u) load_to_lds(pool + t.at[u / (NI / 2)], place[u % (NI / 2)], at + u * 1024);
        } else {
#pragma unroll
            for (int u = 0; u < NI; ++u) {                     // keys outside repeat a valid one: finite values, weight 0
                const int key = u * KPI + lane / PC, src = max(min(t.key0 + key, last), e.t0);
                load_to_lds(pool + t.at[u / (NI / 2)], (uint32_t)((src & (P - 1)) * (D * 2) + ((lane % PC) ^ (key & (PC - 1))) * 16), at + u * 1024);
            }
        }
    };
    // q and the pages arrive before the stream begins: a wait left for the loop would be one for every load under way
    u32x4_t q[RT][KST][QT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = e.r0 + min(t * 16 + col, e.rows - 1), m = r / G;
        const E *p = reinterpret_cast<const E *>(a.q) + (int64_t)(e.seq0 + m) * a.ldq + (h * G + r - m * G) * D + g4 * 8;
#pragma unroll
        for (int ks = 0; ks < KST; ++ks) load_q(p + ks * 32, q[t][ks]);
    }
    Halves now{};
    look_up(0);
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int ks = 0; ks < KST; ++ks)
#pragma unroll
            for (int x = 0; x < QT; ++x) asm volatile("" : "+v"(q[t][ks][x]));
    if (n > 0) { now = halves(0); request(kpool, now, to); request(vpool, now, to + kHalf); }
    const float scale = rsqrtf((float)D) * 1.44269504f;        // scores in units of log2: p is one exp2 instruction
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        M[t] = -INFINITY; den[t] = 0.f;
#pragma unroll
        for (int f = 0; f < FT; ++f) o[t][f] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }
    // the lane's places in K's and V's tiles; a key 16 further on has the same permutation
    const char *kat[KST], *vat[FT];
    {
        const int ka = g4 * 4 + (col >> 2);                    // key whose pieces this lane addresses
#pragma unroll
        for (int ks = 0; ks < KST; ++ks) kat[ks] = ring + (col * PC + ((ks * 4 + g4) ^ (col & (PC - 1)))) * 16;
#pragma unroll
        for (int f = 0; f < FT; ++f) vat[f] = ring + kHalf + (ka * PC + ((f * 2 + ((col & 3) >> 1)) ^ (ka & (PC - 1)))) * 16 + (col & 1) * 8;
    }
    for (int i = 0; i < n; ++i) {
        const int key0 = tb + (i * ws + w0) * kTile;
        wait_newer<NI>();                                      // newer than this tile's K: its V
        u32x4_t kf[2][KST];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int ks = 0; ks < KST; ++ks) kf[j][ks] = *reinterpret_cast<const u32x4_t *>(kat[ks] + j * 16 * PC * 16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // read: the place can be requested anew
        if (i + 1 < n) {
            if (((i + 1) & 31) == 0) look_up(i + 1);
            now = halves(i + 1);
            request(kpool, now, to);
        }
        u32x4_t ph[RT], pm[RT], pl[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            floatx4_t s[QT][2];
#pragma unroll
            for (int x = 0; x < QT; ++x) { s[x][0] = floatx4_t{0.f, 0.f, 0.f, 0.f}; s[x][1] = s[x][0]; }
#pragma unroll
            for (int ks = 0; ks < KST; ++ks)
#pragma unroll
                for (int x = 0; x < QT; ++x)
#pragma unroll
                    for (int j = 0; j < 2; ++j) s[x][j] = mfma_16x16x32(kf[j][ks], q[t][ks][x], s[x][j]);
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = s[0][j >> 2][j & 3];
                if (QT == 3) p[j] += s[QT - 2][j >> 2][j & 3] + s[QT - 1][j >> 2][j & 3];
            }
            if (key0 < e.t0 || key0 + kTile - 1 > last) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = key0 + (j >> 2) * 16 + g4 * 4 + (j & 3);
                    if (key < e.t0 || key > last) p[j] = -INFINITY;
                }
            }
            float mt = p[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) mt = fmaxf(mt, p[j]);
            mt = column_max(mt);
            const float Mn = fmaxf(M[t], mt * scale);
            // Weights are formed in the unit of a maximum seen, not always the last one: up to 2^8 they lose nothing in fp32, and sums are
            // brought to a new unit only where some row's scores pass it by more
            if (__any(Mn > M[t] + 8.f)) {
                const float corr = M[t] == Mn ? 1.f : __builtin_amdgcn_exp2f(M[t] - Mn);     // exp2(-inf) = 0 on the wave's first keys
                M[t] = Mn;
                den[t] *= corr;
#pragma unroll
                for (int f = 0; f < FT; ++f) { o[t][f][0] *= corr; o[t][f][1] *= corr; o[t][f][2] *= corr; o[t][f][3] *= corr; }
            }
            const float m0 = M[t] == -INFINITY ? 0.f : M[t];   // a row whose scores so far all overflowed to -inf: p = 0
#pragma unroll
            for (int j = 0; j < 8; ++j) { p[j] = __builtin_amdgcn_exp2f(fmaf(p[j], scale, -m0)); den[t] += p[j]; }
            if (PT == 3) split3_bf16(p, ph[t], pm[t], pl[t]);
            else split2_bf16(p, ph[t], pm[t]);
        }
        if (i + 1 < n) wait_newer<NI>(); else wait_newer<0>(); // newer than this tile's V: the K requested above
        u32x4_t vf[FT];
#pragma unroll
        for (int f = 0; f < FT; ++f) {
            const uint2 va = lds_read_tr(vat[f]), vb = lds_read_tr(vat[f] + 16 * PC * 16);
            vf[f] = u32x4_t{va.x, va.y, vb.x, vb.y};
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + 1 < n) request(vpool, now, to + kHalf);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
            for (int f = 0; f < FT; ++f) o[t][f] = mfma_16x16x32(vf[f], ph[t], o[t][f]);
#pragma unroll
            for (int f = 0; f < FT; ++f) o[t][f] = mfma_16x16x32(vf[f], pm[t], o[t][f]);
            if (PT == 3) {
#pragma unroll
                for (int f = 0; f < FT; ++f) o[t][f] = mfma_16x16x32(vf[f], pl[t], o[t][f]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        den[t] += __shfl_xor(den[t], 16, 64);
        den[t] += __shfl_xor(den[t], 32, 64);
        if (bad) den[t] = NAN;                                 // a page that the cache does not have: the row's result is no number
    }
    return bad;
}

template <int D, int RT, bool F32>
__device__ __forceinline__ void item(const SharedArgs &a, const SharedRecord &e, int h, bool together, bool once, char *lds, float (*wml)[kSharedRows][2])
{
    constexpr int FT = D / 16, kRing = kTile * D * 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g4 = lane >> 4;
    const int G = a.hq / a.hkv;
    char *ring = lds + wave * kRing;
    floatx4_t o[RT][FT];
    float M[RT], den[RT];
    stream_keys<D, RT, F32>(a, e, h, together ? wave : 0, together ? kW : 1, ring, once, o, M, den);
    if (!together) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (t * 16 + col >= e.rows) continue;
            const int r = e.r0 + t * 16 + col, m = r / G;
            const int64_t row = (int64_t)(e.part0 + m) * a.hq + h * G + r - m * G;
#pragma unroll
            for (int f = 0; f < FT; ++f)
                *reinterpret_cast<float4 *>(a.part_acc + row * D + f * 16 + g4 * 4) = make_float4(o[t][f][0], o[t][f][1], o[t][f][2], o[t][f][3]);
            if (g4 == 0) *reinterpret_cast<float2 *>(a.part_ml + row * 2) = make_float2(M[t], den[t]);
        }
        return;
    }
    // the waves' states meet in LDS (a wave's tiles are read: its ring is free) and are combined in wave order
    static_assert(RT * 16 * D * 4 <= kRing, "a wave's sums fit its ring");
    float *red = reinterpret_cast<float *>(ring);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int f = 0; f < FT; ++f) *reinterpret_cast<float4 *>(red + (t * 16 + col) * D + f * 16 + g4 * 4) = make_float4(o[t][f][0], o[t][f][1], o[t][f][2], o[t][f][3]);
        if (g4 == 0) { wml[wave][t * 16 + col][0] = M[t]; wml[wave][t * 16 + col][1] = den[t]; }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < e.rows * (D / 4); x += kW * 64) {
        const int lr = x / (D / 4), r = e.r0 + lr, m = r / G;
        float mw[kW], Mc = -INFINITY;
#pragma unroll
        for (int w = 0; w < kW; ++w) { mw[w] = wml[w][lr][0]; Mc = fmaxf(Mc, mw[w]); }
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            const float sw = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[w] - Mc);     // a wave without tiles, or whose scores all are -inf
            const float4 t = reinterpret_cast<const float4 *>(lds + w * kRing)[x];
            v.x = fmaf(t.x, sw, v.x); v.y = fmaf(t.y, sw, v.y); v.z = fmaf(t.z, sw, v.z); v.w = fmaf(t.w, sw, v.w);
            l = fmaf(wml[w][lr][1], sw, l);
        }
        const int64_t row = (int64_t)(e.part0 + m) * a.hq + h * G + r - m * G;
        reinterpret_cast<float4 *>(a.part_acc + row * D)[x % (D / 4)] = v;
        if (x % (D / 4) == 0) *reinterpret_cast<float2 *>(a.part_ml + row * 2) = make_float2(Mc, l);
    }
    __syncthreads();                                           // the rings are free for the next item
}

__device__ __forceinline__ bool made_for(const SharedHeader *h, const SharedArgs &a)
{
    return h->mark == kSharedMark && h->n_seqs == a.n_seqs && h->hkv == a.hkv && h->G * h->hkv == a.hq;
}

template <int D, bool F32>
__global__ __launch_bounds__(kW * 64, 2) void attn_shared_kernel(SharedArgs a)
{
    extern __shared__ __align__(16) char lds[];                // [wave][K | V] tiles
    __shared__ float wml[kW][kSharedRows][2];
    const SharedHeader *head = reinterpret_cast<const SharedHeader *>(a.plan);
    const SharedRecord *recs = reinterpret_cast<const SharedRecord *>(reinterpret_cast<const SharedSeq *>(head + 1) + a.n_seqs);
    if (!made_for(head, a)) return;
    const int np = head->n_prefix, no = head->n_own, solo = head->solo, hkv = a.hkv, per = solo ? hkv / kW : hkv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first_own = (int64_t)np * hkv, items = first_own + (int64_t)no * per;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const bool prefix = it < first_own;
        const uint32_t x = (uint32_t)(prefix ? it : it - first_own), div = prefix ? hkv : per, ri = x / div;
        const bool together = prefix || !solo;
        const int h = (int)(x - ri * div) * (together ? 1 : kW) + (together ? 0 : wave);
        const SharedRecord *rp = recs + (prefix ? ri : np + ri);
        SharedRecord e;
        e.seq0 = __builtin_amdgcn_readfirstlane(rp->seq0); e.r0 = __builtin_amdgcn_readfirstlane(rp->r0); e.rows = __builtin_amdgcn_readfirstlane(rp->rows);
        e.table_row = __builtin_amdgcn_readfirstlane(rp->table_row); e.t0 = __builtin_amdgcn_readfirstlane(rp->t0); e.cnt = __builtin_amdgcn_readfirstlane(rp->cnt);
        e.part0 = __builtin_amdgcn_readfirstlane(rp->part0);
        if constexpr (F32) {
            // fp32 queries, three terms each, leave registers for one row tile of 16: the second reads the keys again, from L2
            const int rows = e.rows;
            for (int r = 0; r < rows; r += 16, e.r0 += 16) {
                e.rows = min(16, rows - r);
                item<D, 1, true>(a, e, h, together, !prefix && rows <= 16, lds, wml);
            }
        }
        else if (e.rows <= 16) item<D, 1, F32>(a, e, h, together, !prefix, lds, wml);
        else item<D, 2, F32>(a, e, h, together, !prefix, lds, wml);
    }
}

// ---- the join ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = f32_to_bf16(v); }

// W waves per (sequence, query head), wave w the parts w, w + W, ..: lane i holds features i and, of 128, i + 64.  Of the waves' sums, met in LDS, the
// first makes the result, in their order.
template <int D, int W, typename E>
__global__ __launch_bounds__(W > 4 ? W * 64 : 256) void attn_join_kernel(SharedArgs a)
{
    constexpr int N = D / 64, kTogether = 8, kRows = W > 4 ? 1 : 4 / W;
    static_assert(W == 1 || W > 4, "rows of a workgroup");
    __shared__ float red[W][N + 1][W > 1 ? 64 : 1];
    const int lane = threadIdx.x & 63, wave = W > 1 ? (int)(threadIdx.x >> 6) : 0;
    const int64_t row = (int64_t)blockIdx.x * kRows + (W > 1 ? 0 : threadIdx.x >> 6);
    if (row >= (int64_t)a.n_seqs * a.hq) return;
    const int s = (int)(row / a.hq), hd = (int)(row - (int64_t)s * a.hq);
    const SharedHeader *head = reinterpret_cast<const SharedHeader *>(a.plan);
    SharedSeq q = reinterpret_cast<const SharedSeq *>(head + 1)[s];
    q.bad |= !made_for(head, a);
    E *out = reinterpret_cast<E *>(a.out) + (int64_t)s * a.ldo + (int64_t)hd * D + lane;
    const int n = q.pn + q.sn;
    if (q.bad || n == 0) {                                     // no keys: zero; a length that makes no sense: no number
        const float v = q.bad ? NAN : 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (wave == 0) put(out + i * 64, v);
        return;
    }
    auto part = [&](int i) { return (int64_t)(i < q.pn ? q.p0 + i * q.p_step : q.s0 + i - q.pn) * a.hq + hd; };
    float M = -INFINITY;
    for (int i = lane; i < n; i += 64) M = fmaxf(M, a.part_ml[part(i) * 2]);
    M = wave_max(M);
    float acc[N] = {}, l = 0.f;
    for (int i0 = wave; i0 < n; i0 += 64 * W) {                // lane j: weight of the wave's j-th part from here
        float w = 0.f;
        if (i0 + lane * W < n) {
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + part(i0 + lane * W) * 2);
            w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
            l = fmaf(ml.y, w, l);
        }
        const int m = min(64, (n - i0 + W - 1) / W);
        for (int i = 0; i < m; i += kTogether) {               // loads of several parts on their way; one behind the last repeats it and is left out
            float v[kTogether][N];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const float *p = a.part_acc + part(i0 + min(i + j, m - 1) * W) * D + lane;
#pragma unroll
                for (int k = 0; k < N; ++k) v[j][k] = p[k * 64];
            }
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const float wj = __shfl(w, i + j, 64);
                if (i + j < m) {
#pragma unroll
                    for (int k = 0; k < N; ++k) acc[k] = fmaf(v[j][k], wj, acc[k]);
                }
            }
        }
    }
    l = wave_sum(l);
    if constexpr (W > 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) red[wave][k][lane] = acc[k];
        red[wave][N][lane] = l;
        __syncthreads();
        if (wave) return;
        for (int w = 1; w < W; ++w) {
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] += red[w][k][lane];
            l += red[w][N][lane];
        }
    }
    const float inv = 1.0f / l;
#pragma unroll
    for (int k = 0; k < N; ++k) put(out + k * 64, acc[k] * inv);
}

template <int D, bool F32>
hipError_t launch_shared(const SharedArgs &a, int n_cu, hipStream_t s)
{
    typedef typename std::conditional<F32, float, uint16_t>::type E;
    const int G = a.hq / a.hkv;
    const int64_t items = shared_records(a.n_seqs, G) * a.hkv;
    const unsigned grid = (unsigned)(items < 16 * n_cu ? items : 16 * n_cu);       // by the plan's room: how many items it has is known on the device alone
    attn_shared_kernel<D, F32><<<grid, kW * 64, kW * kTile * D * 4, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // few rows may have many parts each (32 rows of 133 parts: 17 us by a wave alone), many rows have few
    const int64_t rows = (int64_t)a.n_seqs * a.hq;
    if (rows <= 512) attn_join_kernel<D, 8, E><<<(unsigned)rows, 512, 0, s>>>(a);
    else attn_join_kernel<D, 1, E><<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_plan(const SharedPlanArgs &a, hipStream_t s)
{
    attn_plan_kernel<<<1, kPlan, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_attn_shared(const SharedArgs &a, int d, bool f32, int n_cu, hipStream_t s)
{
    if (d == 128) return f32 ? launch_shared<128, true>(a, n_cu, s) : launch_shared<128, false>(a, n_cu, s);
    return f32 ? launch_shared<64, true>(a, n_cu, s) : launch_shared<64, false>(a, n_cu, s);
}

}  // namespace pat
