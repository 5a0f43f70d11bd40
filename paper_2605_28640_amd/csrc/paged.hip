// Dense attention of the newest tokens of many sequences over a pool of pages, the pages that neighbours of the list have in
// common read once for all of them (Eq. 4 with every token).
//
// Mathematics.  With z_j = scale q . k_j and any split of the positions into parts, each part leaves m = max z_j, l = sum e^(z_j - m),
// o = sum e^(z_j - m) v_j, and parts join by m = max m_i, (l, o) = sum e^(m_i - m) (l_i, o_i): the shared pages are one
// part, attended by the rows of all sequences of the run at once, a sequence's own pages another, and each is split
// further along its keys for balance.
//
// Work.  Segments (a run's shared pages, a sequence's own pages) times tiles of query rows, each cut into units of 128 (float32: 64) keys;
// per KV head the units of all segments form one line, the lines of the heads another, and every workgroup takes an equal
// share of it, whatever the lengths are.  Where that line is cut and which unit belongs to whom follows from the lengths alone: each workgroup
// works it out for itself (a prefix sum over the list), so lengths live on the device and nothing has to be planned by the host.
// What a workgroup holds of a tile goes to one of its two boundary records if the tile goes on elsewhere, to the row's record
// if it has a second part (shared and own), else straight to the output; a second launch joins the records.
//
// Two kinds of tile:
//   few rows (at most 32: a sequence's heads at decode): bound by the bytes of K and V.  A workgroup's four waves take 32 keys (float32: 16) each
//     of a unit, every wave by itself: no barrier, its own softmax state, joined at the end of the tile.  K goes
//     from memory into registers in the matrix operand's own layout, V through a wave's own LDS tile; while one is used the other is on its way.
//   many rows (tiles of 128; bfloat16): bound by the matrix units.  Every wave takes 32 rows, all four go through the same keys, K
//     and V tiles in a ring of three LDS slots filled two steps ahead, one barrier a step.
// In both S^T = K Q^T and O^T = V^T P^T, so that a lane holds the keys of one query and P^T goes from the accumulators into the
// second product as it is.
#include <type_traits>

#include "check.h"
#include "common.h"

namespace rs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
constexpr int kMaxList = 1024;
#define PAGED_OCC 2
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // the softmax's reference point moves when the maximum has grown by more (base-2 exponent)

constexpr int kFew = 32, kMany = 128;  // rows of a tile
constexpr int kPartUnits = 1;          // what beginning and ending a tile costs, in units of keys

// keys a wave takes at a time
template <typename ST>
constexpr int kKeys = sizeof(ST) == 2 ? 32 : 16;

struct PagedParams {
    const void *q, *k, *v;
    const int32_t *table, *len, *seq, *n_new, *share;
    void *out;
    float *lse;
    float *cut_o, *cut_ml;      // boundary records: [2 workgroups][cut_rows] x D, x 2
    float *row_o, *row_ml;      // row records: [shared, own][B Hq T] x D, x 2; nullptr: no segment is shared
    char *plan;                 // the first workgroup's plan, for the join
    int B, Hq, Hkv, G, S, M, N, shift, T, groups;
    int own_rows, cut_rows;     // rows of a tile of one sequence, of a boundary record
    float scale;
};

// The line of units of one KV head.
struct Seq {
    int L, n, c, first;  // tokens, new ones, pages of the run's shared part (0: none), the run's first place
};
// A tile of n units takes kPartUnits + n places of the line, the first of them empty; a tile without units none.
__device__ __forceinline__ int places(int n) { return n > 0 ? n + kPartUnits : 0; }
struct Plan {
    Seq *seq;      // [B]
    int *start;    // [B + 1] places of the line before this entry of the list
    int *members;  // [B] members of the run that begins here (0: none begins, or it shares nothing)
    int *fewest;   // [B] pages a run can share
    int *row;      // [B] the sequence's row of the table
    __device__ __forceinline__ Plan(char *at, int B) : seq((Seq *)at), start((int *)(seq + B)), members(start + B + 1), fewest(members + B), row(fewest + B) {}
};
static size_t plan_bytes(int B) { return (size_t)B * 16 + (size_t)(4 * B + 1) * 4; }

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }

// units of row tile rt of sequence x over its own pages: the keys from the shared ones to the tile's last row
template <int UNIT>
__device__ __forceinline__ int own_units(const Seq &x, int rt, int rows, int G, int shift, int &k0, int &k1)
{
    const int t0 = rt * rows / G, t1 = min(x.n - 1, (rt * rows + rows - 1) / G);
    k0 = x.c << shift;
    k1 = x.L - x.n + t1 + 1;
    return (t0 >= x.n || k1 <= k0) ? 0 : (k1 - k0 + UNIT - 1) / UNIT;
}
// rows of a tile of a run's shared part, and its tiles
template <typename ST>
__device__ __forceinline__ int shared_rows(int rows) { return sizeof(ST) == 2 && rows > kFew ? kMany : kFew; }

// Fills the plan; called by the whole workgroup.
template <typename ST>
__device__ __forceinline__ void make_plan(const PagedParams &a, const Plan &pl)
{
    constexpr int UNIT = kPagedWaves * kKeys<ST>;
    const int tid = threadIdx.x;
    for (int b = tid; b < a.B; b += kPagedThreads) {
        const int s = a.seq[b];
        int L = (s >= 0 && s < a.S) ? a.len[s] : 0, n = a.n_new ? a.n_new[b] : a.T;
        L = L < 0 ? 0 : min(L, a.M << a.shift);
        n = n < 0 ? 0 : min(n, a.T);
        int first = b, c = 0;
        if (a.share) {
            const int f = a.share[3 * b];
            if (f >= 0 && f <= b) {
                const int cnt = a.share[3 * f + 1];
                if (a.share[3 * f] == f && cnt > b - f && cnt <= a.B - f && cnt > 1) {
                    first = f;
                    c = min(max(a.share[3 * f + 2], 0), max(L - n, 0) >> a.shift);
                }
            }
        }
        pl.seq[b] = Seq{L, n, c, first};
        pl.members[b] = (c > 0 && first == b) ? a.share[3 * b + 1] : 0;
        pl.fewest[b] = 0x7fffffff;
        pl.row[b] = s;
    }
    __syncthreads();
    if (a.share) {
        for (int b = tid; b < a.B; b += kPagedThreads) atomicMin(&pl.fewest[pl.seq[b].first], pl.seq[b].c);
        __syncthreads();
    }
    // (a thread's stretch of the list, so that a second pass can add what precedes it)
    const int each = div_up(a.B, kPagedThreads), lo = min(tid * each, a.B), hi = min(lo + each, a.B);
    int sum = 0;
    for (int b = lo; b < hi; ++b) {
        Seq x = pl.seq[b];
        x.c = pl.members[x.first] ? pl.fewest[x.first] : 0;  // (nobody writes members, fewest or first here)
        int units = 0, k0, k1;
        if (x.first == b && x.c > 0) {
            const int rows = pl.members[b] * a.T * a.G;
            units += div_up(rows, shared_rows<ST>(rows)) * places(div_up(x.c << a.shift, UNIT));
        }
        for (int rt = 0; rt * a.own_rows < x.n * a.G; ++rt) units += places(own_units<UNIT>(x, rt, a.own_rows, a.G, a.shift, k0, k1));
        pl.start[b] = units;
        pl.seq[b].c = x.c;
        sum += units;
    }
    // what precedes the stretch
    __shared__ int tot[kPagedWaves];
    int inc = sum;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(inc, d, kWave);
        if (lane_id() >= d) inc += o;
    }
    if (lane_id() == kWave - 1) tot[tid >> 6] = inc;
    __syncthreads();
    int at = inc - sum;
    for (int w = 0; w < (tid >> 6); ++w) at += tot[w];
    for (int b = lo; b < hi; ++b) {
        const int u = pl.start[b];
        pl.start[b] = at;
        at += u;
    }
    if (hi == a.B && lo < hi) pl.start[a.B] = at;
    __syncthreads();
}

// Workgroup w of `groups` (no more than there are places) has the places [share_begin(w), share_begin(w + 1)) of the whole line.
__device__ __forceinline__ long share_begin(long w, long all, int groups) { return w * all / groups; }
__device__ __forceinline__ long owner_of(long place, long all, int groups) { return ((place + 1) * groups - 1) / all; }
// where the part of a tile (its units at s0 .. s1 - 1) that lies in [wb, we) goes: 2: all of it is there; 0, 1: a boundary record
__device__ __forceinline__ int record_of(long s0, long s1, long wb, long we) { return (s0 >= wb && s1 <= we) ? 2 : s0 <= wb ? 0 : 1; }

// the last entry of the list that begins at or before off (entries without units are passed over)
__device__ __forceinline__ int place_of(const Plan &pl, int B, int off)
{
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pl.start[mid] <= off) lo = mid;
        else hi = mid;
    }
    return lo;
}

// one tile of rows over a run of keys
struct TileWork {
    int kvh, b, rt, rows;     // rows: of the segment (the tile takes those from rt * tile_rows on)
    int tile_rows;
    bool shared;
    int row_seq;              // whose table row names the pages
    int key0, units, limit;   // first key, units of keys from there, keys that exist (later ones are nobody's)
    int record;               // record_of()
    long slot;                // of the boundary record
    bool direct;              // a whole tile without a second part
    int entries;              // this lane's first entry of the table (PageList)
};

// the tile that place `at` of the whole line belongs to; its units are those at s0 .. s1 - 1
template <typename ST>
__device__ __forceinline__ void find_tile(const PagedParams &a, const Plan &pl, long at, int line, TileWork &w, long &s0, long &s1)
{
    constexpr int UNIT = kPagedWaves * kKeys<ST>;
    w.kvh = (int)(at / line);
    int off = (int)(at % line), n;
    const int lo = w.b = place_of(pl, a.B, off);
    off -= pl.start[lo];
    const Seq x = pl.seq[lo];
    w.row_seq = pl.row[lo];
    int su = 0, st = 0;
    if (x.first == lo && x.c > 0) {
        w.rows = pl.members[lo] * a.T * a.G;
        w.tile_rows = shared_rows<ST>(w.rows);
        n = div_up(x.c << a.shift, UNIT);
        su = places(n);
        st = div_up(w.rows, w.tile_rows);
    }
    w.key0 = 0;
    w.shared = off < su * st;
    if (w.shared) {
        w.rt = off / su;
        off -= w.rt * su;
        w.limit = x.c << a.shift;
    } else {
        off -= su * st;
        w.rt = 0;
        w.rows = x.n * a.G;
        w.tile_rows = a.own_rows;
        for (;; ++w.rt) {
            n = own_units<UNIT>(x, w.rt, a.own_rows, a.G, a.shift, w.key0, w.limit);
            if (off < places(n)) break;
            off -= places(n);
        }
    }
    s0 = at - off + kPartUnits;
    s1 = s0 + n;
}

// the query behind row r of a segment; false: none
__device__ __forceinline__ bool query_of(const PagedParams &a, const Plan &pl, const TileWork &w, int r, int &bq, int &t, int &g)
{
    if (r >= w.rows) return false;
    const int per = a.T * a.G;
    bq = w.b;
    if (w.shared) {
        bq += r / per;
        r %= per;
    }
    t = r / a.G;
    g = r % a.G;
    return t < pl.seq[bq].n;
}
__device__ __forceinline__ long out_row(const PagedParams &a, const TileWork &w, int bq, int t, int g)
{
    return (long)(bq * a.Hq + w.kvh * a.G + g) * a.T + t;
}

// 4 channels (from c) of a row's finished output, or its part of (o, m, l)
template <typename ST, int D>
__device__ __forceinline__ void put4(const PagedParams &a, const TileWork &w, long row, int r, int c, const f32x4 &o, float m, float l)
{
    if (w.direct) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        ST y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) from_f32(y[j], o[j] * inv);
        __builtin_memcpy(__builtin_assume_aligned((ST *)a.out + row * D + c, 4 * sizeof(ST)), y, sizeof(y));
        if (a.lse && c == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
        return;
    }
    const bool whole = w.record == 2;
    const long at = whole ? (w.shared ? 0 : (long)a.B * a.Hq * a.T) + row : w.slot * a.cut_rows + r;
    *reinterpret_cast<f32x4 *>((whole ? a.row_o : a.cut_o) + at * D + c) = o;
    if (c == 0) *reinterpret_cast<float2 *>((whole ? a.row_ml : a.cut_ml) + at * 2) = make_float2(m, l);
}

// ---- pages -----------------------------------------------------------------------------------------------------
// Which rows hold a wave's keys, 16 at a time (a page is 16 keys and more): entry n is that of keys first + (n / PER) * stride +
// 16 (n % PER).  64 entries of the table at a time, one a lane.
template <int PER>
struct PageList {
    const int32_t *row;
    int first, stride, last, limit, N, shift, listed;
    __device__ __forceinline__ int key(int n) const { return first + n / PER * stride + n % PER * 16; }
    // this lane's entry of the 64 from n on, as the table has it
    __device__ __forceinline__ int fetch(int n) const
    {
        const int m = n + lane_id(), k = key(m);
        int page = -1;
        if (m < last && k < limit) page = row[k >> shift];
        return page;
    }
    __device__ __forceinline__ void take(int page)
    {
        listed = (page < 0 || page >= N) ? -1 : page;
        asm volatile("" : "+v"(listed));  // (waited for here, and not by every step)
    }
    // before the first entry of a step after the first is asked for (64 % PER == 0): all lanes
    __device__ __forceinline__ void fill(int n)
    {
        if ((n & 63) == 0) take(fetch(n));
    }
    // rows that exist (0 .. 16), and the first of them
    __device__ __forceinline__ int rows(int n, long &at) const
    {
        const int page = __builtin_amdgcn_readlane(listed, n & 63), k = key(n), left = limit - k;
        at = page < 0 ? 0l : ((long)page << shift) + (k & ((1 << shift) - 1));
        // (a scalar, which the compiler does not see in the clamp: the descriptors made of it would be a loop over the lanes each)
        return __builtin_amdgcn_readfirstlane(page < 0 || left < 0 ? 0 : left < 16 ? left : 16);
    }
};

// the lists of the two kinds of tile
template <typename ST>
__device__ __forceinline__ PageList<kKeys<ST> / 16> few_pages(const PagedParams &a, const TileWork &w)
{
    constexpr int KT = kKeys<ST>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return PageList<KT / 16>{a.table + (long)w.row_seq * a.M, w.key0 + wave * KT, kPagedWaves * KT, w.units * (KT / 16), w.limit, a.N, a.shift, -1};
}
__device__ __forceinline__ PageList<2> many_pages(const PagedParams &a, const TileWork &w)
{
    const int end = min(w.limit, w.key0 + w.units * (kPagedWaves * 32));
    return PageList<2>{a.table + (long)w.row_seq * a.M, w.key0, 32, 2 * ((end - w.key0 + 31) / 32), w.limit, a.N, a.shift, -1};
}

__device__ __forceinline__ s16x4 paged_read_tr16(const char *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}

// max / sum with the lanes 16, 32 and 48 away
__device__ __forceinline__ float quad_max(float x)
{
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return half_pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float x)
{
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return half_pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void pin()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// the LDS of a workgroup: six tiles of 32 bfloat16 (16 float32) rows
struct Ring {
    char *k0, *k1, *k2, *v0, *v1, *v2;
};

// whether any of `chunks` 16-byte pieces of LDS holds an infinity or NaN; every step-th from at on
template <typename ST>
__device__ __forceinline__ bool not_finite(const char *lds, int at, int step, int chunks)
{
    bool odd = false;
#pragma unroll 1
    for (int c = at; c < chunks; c += step) {
        const uint4 x = *reinterpret_cast<const uint4 *>(lds + 16 * c);
        for (const uint32_t u : {x.x, x.y, x.z, x.w}) {
            odd |= (u & 0x7f800000u) == 0x7f800000u;
            if (sizeof(ST) == 2) odd |= (u & 0x7f80u) == 0x7f80u;
        }
    }
    return odd;
}

// The same tile key by key, only the keys that a row sees: where V holds an infinity or NaN that some row is not to see, and
// a matrix product would take 0 times it.  D / 4 lanes a row.
template <typename ST, int D>
__device__ __forceinline__ void attend_by_key(const PagedParams &a, const Plan &pl, const TileWork &w)
{
    constexpr int UNIT = kPagedWaves * kKeys<ST>, C4 = D / 4, NG = kPagedThreads / C4;
    const int c4 = threadIdx.x % C4, end = min(w.limit, w.key0 + w.units * UNIT);
    const int32_t *pages = a.table + (long)w.row_seq * a.M;
    const long pool = (long)w.kvh * ((long)a.N << a.shift);
    const float cs = a.scale * kLog2e;
    for (int r = threadIdx.x / C4; r < w.tile_rows; r += NG) {
        int bq, t, g;
        if (!query_of(a, pl, w, w.rt * w.tile_rows + r, bq, t, g)) continue;
        const long row = out_row(a, w, bq, t, g);
        const int last = w.shared ? end - 1 : min(end - 1, pl.seq[bq].L - pl.seq[bq].n + t);
        float q[4], m = -INFINITY, l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = to_f32(((const ST *)a.q)[row * D + 4 * c4 + j]);
        for (int key = w.key0; key <= last; ++key) {
            const int page = pages[key >> a.shift];
            if (page < 0 || page >= a.N) continue;
            const long at = (pool + ((long)page << a.shift) + (key & ((1 << a.shift) - 1))) * D + 4 * c4;
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) z = fmaf(q[j], to_f32(((const ST *)a.k)[at + j]), z);
            z = group_sum<C4>(z) * cs;
            const float top = fmaxf(m, z), f = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), p = z == top ? 1.f : __builtin_amdgcn_exp2f(z - top);
            m = top;
            l = l * f + p;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = o[j] * f + p * to_f32(((const ST *)a.v)[at + j]);
        }
        put4<ST, D>(a, w, row, r, 4 * c4, o, m, l);
    }
    __syncthreads();
}

// ---- few rows --------------------------------------------------------------------------------------------------
// 16-wide matrix instructions: lane (l16, lg) = (lane % 16, lane / 16) holds query l16 and, of every 16 keys, 4 lg .. 4 lg + 3.
// K operand: row l16, 16 bytes at chunk 4 kk + lg, straight from memory (a load touches 64 bytes of each of 16 rows; the lines
// are used up by the loads beside it).  V operand, bfloat16: transpose reads of the row-major tile, chunks of a row
// permuted so that 32 lanes reading two chunks of each of 8 rows touch every bank once; float32: four chunks of each of 4 rows.
template <typename ST, int D>
struct FewRows {
    static constexpr int ROW = D * (int)sizeof(ST), CR = ROW / 16, RW = 64 / CR, NL = 16 / RW;  // chunks a row, rows and loads a wave
    __device__ __forceinline__ static int v_swizzle(int row)
    {
        if (sizeof(ST) == 4) return 4 * ((row >> 2) & 3);
        return CR == 16 ? 2 * (row & 7) : 2 * ((row >> 1) & 3);
    }
    // 16 rows of V from a descriptor that ends with the last valid one into LDS
    __device__ __forceinline__ static void load_v(LdsSource src, char *tile)
    {
        const int lane = lane_id();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = i * RW + lane / CR, chunk = (lane % CR) ^ v_swizzle(row);
            load16_to_lds_at<2>(src, (uint32_t)(row * ROW + chunk * 16), 0u, tile + i * 1024);
        }
    }
};

template <typename ST, int D, int RT>
__device__ __forceinline__ void attend_few(const PagedParams &a, const Plan &pl, const TileWork &w, const Ring &lds, float *s_m, float *s_l)
{
    using Rows = FewRows<ST, D>;
    constexpr bool BF = sizeof(ST) == 2;
    constexpr int KT = kKeys<ST>, NH = KT / 16, ROW = Rows::ROW;
    constexpr int NDT = D / 16, NK = BF ? D / 32 : D / 16;  // 16-channel tiles of O^T; 16-byte operands of a row
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    char *const cV = wave == 0 ? lds.k0 : wave == 1 ? lds.k1 : wave == 2 ? lds.k2 : lds.v0;

    const long pool = (long)w.kvh * ((long)a.N << a.shift);
    const ST *kb = (const ST *)a.k + pool * D, *vb = (const ST *)a.v + pool * D;
    PageList<NH> pages = few_pages<ST>(a, w);
    pages.take(w.entries);

    f32x4 kf[NH][NK];
    LdsSource v_src[NH];
    int valid[NH];
    const uint32_t k_at = (uint32_t)(l16 * ROW + lg * 16);
    auto load_k = [&](int u) __attribute__((always_inline)) {  // also looks up where the step's rows are
        if (u > 0) pages.fill(u * NH);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            long at;
            valid[h] = pages.rows(u * NH + h, at);
            const LdsSource src = lds_source_sized(kb + at * D, valid[h] * ROW);
            v_src[h] = lds_source_sized(vb + at * D, valid[h] * ROW);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                const auto x = __builtin_amdgcn_raw_buffer_load_b128(src, k_at + 64 * kk, 0, 2);
                kf[h][kk] = __builtin_bit_cast(f32x4, x);
            }
        }
        pin();
    };
    auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < NH; ++h) Rows::load_v(v_src[h], cV + h * 16 * ROW);
        pin();
    };
    load_k(0);
    load_v();

    // ---- this lane's queries ----
    f32x4 qf[RT][NK];
    int last[RT];                 // the last position the row sees (-1: there is no such row)
    int first_last = 0x7fffffff;  // the smallest of the tile's rows
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        int bq, t, g;
        const bool real = query_of(a, pl, w, w.rt * w.tile_rows + rt * 16 + l16, bq, t, g);
        last[rt] = -1;
        const ST *q = (const ST *)a.q;
        if (real) {
            q += out_row(a, w, bq, t, g) * D;
            last[rt] = pl.seq[bq].L - pl.seq[bq].n + t;
        }
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const char *>(q) + 64 * kk + 16 * lg);
            qf[rt][kk] = real ? x : f32x4{0.f, 0.f, 0.f, 0.f};
        }
        first_last = min(first_last, last[rt]);
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) first_last = min(first_last, __shfl_xor(first_last, m, kWave));
    first_last = __builtin_amdgcn_readfirstlane(first_last);
    if (w.shared) first_last = 0x7fffffff;  // every row sees all of it (what comes of rows that do not exist is dropped)

    f32x4 oacc[RT][NDT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) oacc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float cs = a.scale * kLog2e;
    // where a lane reads V of the tile's first 16 channels; of 16-channel tile dt: ^ 16 * (chunks of it)
    uint32_t v_at[BF ? 1 : 4];
    if constexpr (BF) {
        const int row = 4 * lg + (l16 >> 2);
        v_at[0] = (uint32_t)(row * ROW + ((((l16 & 3) >> 1) ^ Rows::v_swizzle(row)) * 16) + 8 * (l16 & 1));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v_at[j] = (uint32_t)((4 * lg + j) * ROW + (((l16 >> 2) ^ Rows::v_swizzle(4 * lg + j)) * 16) + 4 * (l16 & 3));
    }

    bool odd = false;  // values that are not finite where some row may not look
#pragma unroll 1
    for (int u = 0; u < w.units; ++u) {
        const int key = w.key0 + wave * KT + u * (kPagedWaves * KT);
        // ---- S^T = K Q^T ----
        f32x4 s[RT][NH];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                s[rt][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < NK; ++kk) {
                    if constexpr (BF) {
                        s[rt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[h][kk]),
                                                                          __builtin_bit_cast(bf16x8, qf[rt][kk]), s[rt][h], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[rt][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[h][kk][j], qf[rt][kk][j], s[rt][h], 0, 0, 0);
                    }
                }
            }
        int here[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) here[h] = valid[h];
        load_k(u + 1);  // (past the last unit: descriptors of no rows)
        // ---- softmax, base 2 ----
        const bool edge = key + KT - 1 > first_last;  // some row does not see some key of this step
        const bool masked = edge || here[0] < 16 || here[NH - 1] < 16;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int h = 0; h < NH; ++h) s[rt][h] *= cs;
        if (masked) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int h = 0; h < NH; ++h)
                {
                    const int sees = min(here[h], edge ? last[rt] + 1 - key - 16 * h : 16) - 4 * lg;  // of the lane's four
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rt][h][i] = i < sees ? s[rt][h][i] : -INFINITY;
                }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = -INFINITY;
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[rt][h][i]);
            mx = quad_max(mx);
            if (__any(mx - m[rt] > kSlack)) {  // (-inf from -inf compares false)
                const float to = (mx - m[rt] > kSlack) ? mx : m[rt];
                const float alpha = (m[rt] == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m[rt] - to);
                l[rt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) oacc[rt][dt] *= alpha;
                m[rt] = to;
            }
            const float bias = (m[rt] == -INFINITY) ? 0.f : m[rt];
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[rt][h][i] = __builtin_amdgcn_exp2f(s[rt][h][i] - bias);
                    l[rt] += s[rt][h][i];
                }
        }
        // ---- O^T += V^T P^T ----
        pin();
        wait_loads<NH * NK>();  // V is here (the next K, issued after it, may be on its way)
        if (edge) odd |= not_finite<ST>(cV, lane, 64, KT * ROW / 16);
        if constexpr (BF) {
            bf16x8 pf[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 8; ++i) pf[rt][i] = (__bf16)s[rt][i / 4][i % 4];
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                union {
                    s16x4 h[2];
                    bf16x8 f;
                } vf;
#pragma unroll
                for (int h = 0; h < 2; ++h) vf.h[h] = paged_read_tr16(cV + (v_at[0] ^ (uint32_t)(32 * dt)) + h * 16 * ROW);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) oacc[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.f, pf[rt], oacc[rt][dt], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float vf = *reinterpret_cast<const float *>(cV + (v_at[j] ^ (uint32_t)(64 * dt)));
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) oacc[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, s[rt][0][j], oacc[rt][dt], 0, 0, 0);
                }
        }
        wait_lds_reads();
        load_v();
    }

    // ---- the four waves' parts become one ----
    wait_loads<0>();  // (nothing lands in this LDS any more)
    if (__syncthreads_or(odd)) return attend_by_key<ST, D>(a, pl, w);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float sum = quad_sum(l[rt]);
        if (lg == 0) {
            s_m[wave * kFew + rt * 16 + l16] = m[rt];
            s_l[wave * kFew + rt * 16 + l16] = sum;
        }
    }
    constexpr int C4 = D / 4;  // 16-byte columns of an output row
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        f32x4 *mine = reinterpret_cast<f32x4 *>(cV);  // 16 rows of D floats: as large as a step's V
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) mine[l16 * C4 + ((4 * dt + lg) ^ l16)] = oacc[rt][dt];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * C4; e += kPagedThreads) {
            const int r = e / C4, c4 = e % C4;
            int bq, t, g;
            if (!query_of(a, pl, w, w.rt * w.tile_rows + rt * 16 + r, bq, t, g)) continue;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kPagedWaves; ++i) top = fmaxf(top, s_m[i * kFew + rt * 16 + r]);
            float L = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kPagedWaves; ++i) {
                const float mi = s_m[i * kFew + rt * 16 + r], li = s_l[i * kFew + rt * 16 + r];
                if (mi == -INFINITY && li == 0.f) continue;  // saw nothing
                const float f = mi == top ? 1.f : __builtin_amdgcn_exp2f(mi - top);
                L = fmaf(f, li, L);
                const char *tile = i == 0 ? lds.k0 : i == 1 ? lds.k1 : i == 2 ? lds.k2 : lds.v0;
                const f32x4 x = *(reinterpret_cast<const f32x4 *>(tile) + r * C4 + (c4 ^ r));
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(f, x[j], o[j]);
            }
            put4<ST, D>(a, w, out_row(a, w, bq, t, g), rt * 16 + r, 4 * c4, o, top, L);
        }
        __syncthreads();
    }
}

// ---- many rows -------------------------------------------------------------------------------------------------
// 32-wide matrix instructions: lane (lq, h) = (lane % 32, lane / 32) holds query lq and keys 8 i + 4 h .. + 3 of a step's 32.
template <int D>
__device__ __forceinline__ void attend_many(const PagedParams &a, const Plan &pl, const TileWork &w, const Ring &lds)
{
    constexpr int NC = D / 16, NDT = D / 32, CR = D / 8, RW = 64 / CR, RPI = kPagedWaves * RW, CPT = 32 / RPI, ROW = 2 * D;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lq = lane & 31, h = lane >> 5;
    const long pool = (long)w.kvh * ((long)a.N << a.shift);
    const bf16 *kb = (const bf16 *)a.k + pool * D, *vb = (const bf16 *)a.v + pool * D;
    PageList<2> pages = many_pages(a, w);
    const int n_steps = pages.last / 2;
    pages.take(w.entries);

    // staging: pass i of a tile: this wave fetches RW rows, rows RPI i + RW wave on, all of one 16-key group
    const int row0 = (RW * wave + lane / CR) & 15;  // in the group
    const uint32_t gk = (uint32_t)(row0 * ROW + (((lane % CR) ^ chunk_swizzle<D>(row0)) * 16));
    const uint32_t gv = (uint32_t)(row0 * ROW + (((lane % CR) ^ chunk_swizzle<D>(row0 & 7)) * 16));
    LdsSource k_src[CPT], v_src[CPT];
    auto look_up = [&](int step) __attribute__((always_inline)) -> int {  // valid rows of the two groups, 8 bits each
        if (step > 0) pages.fill(2 * step);
        long at[2];
        const int r0 = pages.rows(2 * step, at[0]), r1 = pages.rows(2 * step + 1, at[1]);
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const bool second = (RPI * i + RW * wave) >= 16;
            const long x = (second ? at[1] : at[0]) * D;
            k_src[i] = lds_source_sized(kb + x, (second ? r1 : r0) * ROW);
            v_src[i] = lds_source_sized(vb + x, (second ? r1 : r0) * ROW);
        }
        return r0 | r1 << 8;
    };
    auto stage_k = [&](int i, char *tile) __attribute__((always_inline)) { load16_to_lds_at(k_src[i], gk, 0u, tile + (RPI * i + RW * wave) * ROW); };
    auto stage_v = [&](int i, char *tile) __attribute__((always_inline)) { load16_to_lds_at(v_src[i], gv, 0u, tile + (RPI * i + RW * wave) * ROW); };
    int valid0 = look_up(0);
#pragma unroll
    for (int i = 0; i < CPT; ++i) stage_k(i, lds.k0), stage_v(i, lds.v0);
    int valid1 = look_up(1);
#pragma unroll
    for (int i = 0; i < CPT; ++i) stage_k(i, lds.k1), stage_v(i, lds.v1);

    // ---- this lane's query ----
    int bq = 0, t = 0, g = 0;
    const int r = wave * 32 + lq;
    const bool real = query_of(a, pl, w, w.rt * w.tile_rows + r, bq, t, g);
    const long row = real ? out_row(a, w, bq, t, g) : 0;
    const int last = real ? pl.seq[bq].L - pl.seq[bq].n + t : -1;
    bf16x8 qf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>((const bf16 *)a.q + row * D + 16 * c + 8 * h);
        qf[c] = __builtin_bit_cast(bf16x8, real ? x : f32x4{0.f, 0.f, 0.f, 0.f});
    }
    int first_last = last, wave_last = last;  // the smallest and the largest of the wave's rows
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        first_last = min(first_last, __shfl_xor(first_last, x, kWave));
        wave_last = max(wave_last, __shfl_xor(wave_last, x, kWave));
    }
    first_last = __builtin_amdgcn_readfirstlane(first_last);
    wave_last = __builtin_amdgcn_readfirstlane(wave_last);
    if (w.shared) first_last = 0x7fffffff, wave_last = wave_last >= 0 ? 0x7fffffff : -1;
    // the smallest of the tile's rows (later positions are later rows of it)
    const int tile_first = w.shared ? 0x7fffffff : pl.seq[w.b].L - pl.seq[w.b].n + w.rt * kMany / a.G;
    bool odd = false;  // values that are not finite where some row may not look

    // operand addresses inside a tile: K row lq, chunk 2 c + h; V through the transpose read, lane = 32 h + 16 dg + L supplying 8 bytes of row
    // 16 c + 4 h + L / 4 (+ 8 for the second read) at channel 32 dt + 16 dg + 4 (L % 4)
    const int L16 = lane & 15, dg = (lane >> 4) & 1;
    const uint32_t koff = (uint32_t)(lq * ROW + ((h ^ chunk_swizzle<D>(lq)) * 16));
    const int rowa = 4 * h + (L16 >> 2);
    const uint32_t voff = (uint32_t)(rowa * ROW + (((2 * dg + ((L16 & 3) >> 1)) ^ chunk_swizzle<D>(rowa)) * 16) + 8 * (L16 & 1));

    f32x16 oacc[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] = 0.f;
    const float cs = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    wait_loads<2 * CPT>();  // the first tile has landed
    asm volatile("s_barrier" ::: "memory");

    auto step = [&](auto buf_tag, int it) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_tag)::value;
        const char *cK = BUF == 0 ? lds.k0 : BUF == 1 ? lds.k1 : lds.k2, *cV = BUF == 0 ? lds.v0 : BUF == 1 ? lds.v1 : lds.v2;
        char *nK = BUF == 0 ? lds.k2 : BUF == 1 ? lds.k0 : lds.k1, *nV = BUF == 0 ? lds.v2 : BUF == 1 ? lds.v0 : lds.v1;
        const int key = w.key0 + it * 32, here = valid0;
        valid0 = valid1;
        valid1 = look_up(it + 2);  // (past the last step: descriptors of no rows)
        const bool live = key <= wave_last;
        if (key + 31 > tile_first) odd |= not_finite<bf16>(cV, threadIdx.x, kPagedThreads, 32 * ROW / 16);
        if (!live) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) stage_k(i, nK), stage_v(i, nV);
        } else {
            f32x16 s;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = 0.f;
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (c % (NC / CPT) == 0) stage_k(c / (NC / CPT), nK);
                const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(cK + (koff ^ (uint32_t)(32 * c)));
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[c], s, 0, 0, 0);
            }
            // operand reads run three matrix instructions ahead of their use, the direct loads go out in between
            __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
            for (int i = 0; i < NC - 3; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (i < CPT) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);
            __builtin_amdgcn_s_setprio(0);
            const bool edge = key + 31 > first_last;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] *= cs;
            if (edge || here != (16 | 16 << 8)) {
                const int sees0 = min(here & 255, edge ? last + 1 - key : 16) - 4 * h, sees1 = min(here >> 8, edge ? last - 15 - key : 16) - 4 * h;
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v] = (v / 4 % 2 * 8 + v % 4 < (v < 8 ? sees0 : sees1)) ? s[v] : -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
            mx = half_pair_max(mx);
            if (__any(mx - m > kSlack)) {
                const float to = (mx - m > kSlack) ? mx : m;
                const float alpha = (m == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m - to);
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
                m = to;
            }
            const float bias = (m == -INFINITY) ? 0.f : m;
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[v] = __builtin_amdgcn_exp2f(s[v] - bias);
                s4[v % 4] += s[v];
            }
            l += (s4[0] + s4[1]) + (s4[2] + s4[3]);
            auto v_of = [&](int c, int dt, int second) __attribute__((always_inline)) {
                return paged_read_tr16(cV + (voff ^ (uint32_t)(64 * dt)) + (16 * c + 8 * second) * ROW);
            };
            __builtin_amdgcn_s_setprio(1);
            bf16x8 pf[2];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) pf[c][i] = (__bf16)s[8 * c + i];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (c < CPT) stage_v(c, nV);
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    union {
                        s16x4 s[2];
                        bf16x8 f;
                    } vf;
                    vf.s[0] = v_of(c, dt, 0);
                    vf.s[1] = v_of(c, dt, 1);
                    oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.f, pf[c], oacc[dt], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int i = 0; i < 2 * NDT - 3; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                if (i < CPT) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);
            __builtin_amdgcn_s_setprio(0);
        }
        // the next step's tile has landed (the one after it may be on its way), and this wave has read what it needs
        __builtin_amdgcn_s_waitcnt(0x0070 | (2 * CPT));
        asm volatile("s_barrier" ::: "memory");
    };
    for (int it = 0;;) {
        step(std::integral_constant<int, 0>{}, it);
        if (++it >= n_steps) break;
        step(std::integral_constant<int, 1>{}, it);
        if (++it >= n_steps) break;
        step(std::integral_constant<int, 2>{}, it);
        if (++it >= n_steps) break;
    }
    wait_loads<0>();  // (nothing lands in the ring any more)
    if (__syncthreads_or(odd)) return attend_by_key<bf16, D>(a, pl, w);
    const float sum = half_pair_sum(l);
    if (real) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = oacc[dt][4 * i + j];
                put4<bf16, D>(a, w, row, r, 32 * dt + 8 * i + 4 * h, o, m, sum);
            }
    }
}

template <typename ST, int D>
__global__ __launch_bounds__(kPagedThreads, PAGED_OCC) void paged_attend_kernel(const PagedParams a)
{
    constexpr int TILE = kKeys<ST> * D * (int)sizeof(ST);
    __shared__ __attribute__((aligned(1024))) char k0[TILE];
    __shared__ __attribute__((aligned(1024))) char k1[TILE];
    __shared__ __attribute__((aligned(1024))) char k2[TILE];
    __shared__ __attribute__((aligned(1024))) char v0[TILE];
    __shared__ __attribute__((aligned(1024))) char v1[TILE];
    __shared__ __attribute__((aligned(1024))) char v2[TILE];
    __shared__ float s_m[kPagedWaves * kFew], s_l[kPagedWaves * kFew];
    extern __shared__ __attribute__((aligned(16))) char lds_plan[];
    const Ring ring{k0, k1, k2, v0, v1, v2};
    const Plan pl(lds_plan, a.B);
    make_plan<ST>(a, pl);
    if (blockIdx.x == 0) {  // for the join
        const Plan to(a.plan, a.B);
        for (int b = threadIdx.x; b < a.B; b += kPagedThreads) {
            to.seq[b] = pl.seq[b];
            to.start[b] = pl.start[b];
            to.members[b] = pl.members[b];
            to.row[b] = pl.row[b];
        }
        if (threadIdx.x == 0) to.start[a.B] = pl.start[a.B];
    }
    const int line = pl.start[a.B];
    const long all = (long)line * a.Hkv;
    const int groups = (int)min((long)gridDim.x, all);
    // Workgroups are dealt to the eight XCDs in turn: those of one XCD take neighbouring shares of the line, tiles of one KV head
    // as a rule, whose rows they find in their L2; less work than workgroups goes to all XCDs.
    const int me = groups < (int)gridDim.x ? (int)blockIdx.x : (int)(blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8);
    if (me >= groups) return;
    const long wb = share_begin(me, all, groups), we = share_begin(me + 1, all, groups);
    long at = wb;
    // the next part of this workgroup's, with the first entries of its table row on their way
    auto next = [&](TileWork &w) __attribute__((always_inline)) -> bool {
        while (at < we) {
            long s0, s1;
            find_tile<ST>(a, pl, at, line, w, s0, s1);
            const long from = max(at, s0), to = min(we, s1);
            at = s1;
            if (from >= to) continue;  // only the place before the units
            w.key0 += (int)(from - s0) * (kPagedWaves * kKeys<ST>);
            w.units = (int)(to - from);
            w.record = record_of(s0, s1, wb, we);
            w.slot = 2l * me + (w.record & 1);
            w.direct = w.record == 2 && !w.shared && pl.seq[w.b].c == 0;
            if (sizeof(ST) == 2 && w.tile_rows == kMany) w.entries = many_pages(a, w).fetch(0);
            else w.entries = few_pages<ST>(a, w).fetch(0);
            return true;
        }
        return false;
    };
    TileWork w;
    bool more = next(w);
#pragma unroll 1
    while (more) {
        TileWork then;
        more = next(then);
        if (sizeof(ST) == 2 && w.tile_rows == kMany) {
            if constexpr (sizeof(ST) == 2) attend_many<D>(a, pl, w, ring);
        } else if (w.rows - w.rt * kFew <= 16) {
            attend_few<ST, D, 1>(a, pl, w, ring, s_m, s_l);
        } else {
            attend_few<ST, D, 2>(a, pl, w, ring, s_m, s_l);
        }
        w = then;
    }
}

// ---- the join --------------------------------------------------------------------------------------------------
// Records are joined by a workgroup's 4 x 64 / (D / 4) groups of D / 4 threads, 16 bytes of the row a thread.
template <typename ST, int D>
struct Join {
    static constexpr int C4 = D / 4, NG = kPagedThreads / C4;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float m1, float l1, const f32x4 &v)
    {
        if (m1 == -INFINITY && l1 == 0.f) return;  // saw nothing
        const float top = fmaxf(m, m1), f0 = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), f1 = m1 == top ? 1.f : __builtin_amdgcn_exp2f(m1 - top);
        m = top;
        l = l * f0 + l1 * f1;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = o[j] * f0 + v[j] * f1;
    }
    // every step-th record of a tile's row, from the lo-th on: its units are at s0 .. s1 - 1; row r of the tile; whole: its row record
    __device__ __forceinline__ void add_tile(const PagedParams &a, long s0, long s1, long all, int groups, int r, long whole, int lo, int step, int c4)
    {
        const long w0 = owner_of(s0, all, groups), w1 = owner_of(s1 - 1, all, groups);
        for (long w = w0 + lo; w <= w1; w += step) {
            const int rec = record_of(s0, s1, share_begin(w, all, groups), share_begin(w + 1, all, groups));
            const long at = rec == 2 ? whole : (2 * w + rec) * a.cut_rows + r;
            const float2 ml = *reinterpret_cast<const float2 *>((rec == 2 ? a.row_ml : a.cut_ml) + at * 2);
            add(ml.x, ml.y, *reinterpret_cast<const f32x4 *>((rec == 2 ? a.row_o : a.cut_o) + at * D + 4 * c4));
        }
    }
    __device__ __forceinline__ void put(const PagedParams &a, long row, int c4) const
    {
        TileWork w;
        w.direct = true;
        put4<ST, D>(a, w, row, 0, 4 * c4, o, m, l);
    }
};

// Where sequences share pages: every row has its shared and its own part, and at most kMany rows of a sequence are one tile.
template <typename ST, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_join_rows_kernel(const PagedParams a)
{
    constexpr int UNIT = kPagedWaves * kKeys<ST>;
    using J = Join<ST, D>;
    __shared__ float s_m[J::NG], s_l[J::NG];
    __shared__ f32x4 s_o[J::NG][J::C4];
    const Plan pl(a.plan, a.B);
    const int c4 = threadIdx.x % J::C4, grp = threadIdx.x / J::C4;
    const long rows = (long)a.B * a.Hq * a.T;
    const int line = pl.start[a.B];
    const long all = (long)line * a.Hkv;
    const int groups = (int)min((long)a.groups, all);
    for (long row = blockIdx.x; row < rows; row += gridDim.x) {
        const int t = (int)(row % a.T), hq = (int)(row / a.T % a.Hq), b = (int)(row / a.T / a.Hq);
        const Seq x = pl.seq[b];
        if (t >= x.n) continue;
        const int kvh = hq / a.G, g = hq % a.G;
        J j;
        int k0, k1;
        const int own = own_units<UNIT>(x, 0, a.own_rows, a.G, a.shift, k0, k1);
        long s0 = (long)kvh * line + pl.start[b] + kPartUnits;
        if (x.c > 0) {
            const int lead = x.first, su = div_up(x.c << a.shift, UNIT), all_rows = pl.members[lead] * a.T * a.G, tile = shared_rows<ST>(all_rows);
            const int r = ((b - lead) * a.T + t) * a.G + g;
            const long t0 = (long)kvh * line + pl.start[lead] + (long)(r / tile) * places(su) + kPartUnits;
            j.add_tile(a, t0, t0 + su, all, groups, r % tile, row, grp, J::NG, c4);
            if (lead == b) s0 += (long)places(su) * div_up(all_rows, tile);
        } else if (own > 0 && owner_of(s0, all, groups) == owner_of(s0 + own - 1, all, groups)) {
            continue;  // written as it is (the same for the whole workgroup)
        }
        if (own > 0) j.add_tile(a, s0, s0 + own, all, groups, t * a.G + g, rows + row, J::NG - 1 - grp, J::NG, c4);
        if (c4 == 0) {
            s_m[grp] = j.m;
            s_l[grp] = j.l;
        }
        s_o[grp][c4] = j.o;
        __syncthreads();
        if (grp == 0) {
            J sum;
#pragma unroll
            for (int i = 0; i < J::NG; ++i) sum.add(s_m[i], s_l[i], s_o[i][c4]);
            sum.put(a, row, c4);
        }
        __syncthreads();
    }
}

// Where they do not: only the tiles that the line's cuts go through, workgroup i looking at the end of the i-th share; and the rows that see
// nothing, which may have no tile.
template <typename ST, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_join_cuts_kernel(const PagedParams a)
{
    using J = Join<ST, D>;
    const Plan pl(a.plan, a.B);
    const int c4 = threadIdx.x % J::C4, grp = threadIdx.x / J::C4;
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int none = min(pl.seq[b].n - pl.seq[b].L, pl.seq[b].n);
        for (int e = grp; e < none * a.Hq; e += J::NG) {
            J j;
            j.put(a, (long)(b * a.Hq + e / none) * a.T + e % none, c4);
        }
    }
    const int line = pl.start[a.B];
    const long all = (long)line * a.Hkv;
    const int groups = (int)min((long)a.groups, all);
    if ((int)blockIdx.x + 1 >= groups) return;
    const long cut = share_begin(blockIdx.x + 1, all, groups);
    TileWork w;
    long s0, s1;
    find_tile<ST>(a, pl, cut, line, w, s0, s1);
    if (cut <= s0 || share_begin(blockIdx.x, all, groups) > s0) return;  // not through its units; not its first
    const int rows = min(w.rows - w.rt * w.tile_rows, w.tile_rows);
    for (int r = grp; r < rows; r += J::NG) {
        int bq, t, g;
        w.shared = false;
        if (!query_of(a, pl, w, w.rt * w.tile_rows + r, bq, t, g)) continue;
        J j;
        j.add_tile(a, s0, s1, all, groups, r, 0, 0, 1, c4);
        j.put(a, out_row(a, w, bq, t, g), c4);
    }
}

int check_pool(const rs_pool *p);  // pool.hip

constexpr int kPagedGroups = 256 * PAGED_OCC;

static bool many_rows(const rs_shape *s, long rows) { return s->dtype == RS_BF16 && rows > kFew; }
static int unit_keys(int dtype) { return kPagedWaves * (dtype == RS_BF16 ? kKeys<bf16> : kKeys<float>); }

// Whether the rows of several sequences are put together: only where one sequence's rows leave room in a tile; else a
// tile's rows come from one sequence anyway and its keys are one segment, without records to join.
static bool rows_are_shared(const rs_shape *s, int T_new) { return (long)T_new * (s->Hq / s->Hkv) < (s->dtype == RS_BF16 ? kMany : kFew); }

struct PagedLayout {
    size_t cut, rows, off_ml, off_plan, total;  // records of each kind
};
static PagedLayout paged_layout(const rs_shape *s, int T_new)
{
    PagedLayout x;
    const long most = rows_are_shared(s, T_new) ? (long)s->B * T_new * (s->Hq / s->Hkv) : (long)T_new * (s->Hq / s->Hkv);
    x.cut = (size_t)2 * kPagedGroups * (many_rows(s, most) ? kMany : kFew);
    x.rows = rows_are_shared(s, T_new) ? (size_t)s->B * s->Hq * T_new * 2 : 0;
    x.off_ml = RS_WS_CTRL_BYTES + align256((x.cut + x.rows) * s->D * 4);
    x.off_plan = x.off_ml + align256((x.cut + x.rows) * 8);
    x.total = x.off_plan + align256(plan_bytes(s->B));
    return x;
}

static int check_paged(const rs_shape *s, const rs_pool *p, int T_new)
{
    int st = check_shape(s, true);
    if (st == RS_OK) st = check_pool(p);
    if (st != RS_OK) return st;
    if (p->P != s->P || (long)p->N * p->P != s->Tcap || T_new < 1) return RS_INVALID_ARG;
    if (s->B > kMaxList) return RS_UNSUPPORTED;
    // units of a KV head's line, at most: they are counted in 32 bits
    const double tiles = (double)s->B * ((double)T_new * (s->Hq / s->Hkv) / kFew + 2);
    if (tiles * ((double)p->M * p->P / unit_keys(s->dtype) + 1) * 2 > 2e9 || (double)s->B * s->Hq * T_new > 2e9) return RS_UNSUPPORTED;
    return RS_OK;
}

template <typename ST, int D>
static void paged_launch(const PagedParams &a, hipStream_t stream)
{
    paged_attend_kernel<ST, D><<<(unsigned)a.groups, kPagedThreads, plan_bytes(a.B), stream>>>(a);
    const long rows = (long)a.B * a.Hq * a.T;
    if (a.share) paged_join_rows_kernel<ST, D><<<(unsigned)(rows < 2048 ? rows : 2048), kPagedThreads, 0, stream>>>(a);
    else paged_join_cuts_kernel<ST, D><<<(unsigned)a.groups, kPagedThreads, 0, stream>>>(a);
}

}  // namespace rs

using namespace rs;

extern "C" {

size_t attn_paged_workspace_bytes(const rs_shape *s, const rs_pool *p, int32_t T_new)
{
    return check_paged(s, p, T_new) == RS_OK ? paged_layout(s, T_new).total : 0;
}

int32_t attn_paged(const rs_shape *s, const rs_pool *p, const void *q, const void *k_pool, const void *v_pool, const int32_t *table,
                   const int32_t *len, const int32_t *seq, const int32_t *n_new, int32_t T_new, const int32_t *share, float scale, void *out,
                   float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_paged(s, p, T_new);
    if (st != RS_OK) return st;
    if (!q || !k_pool || !v_pool || !table || !len || !seq || !out) return RS_INVALID_ARG;
    for (const void *x : {q, k_pool, v_pool, (const void *)table, (const void *)len, (const void *)seq, (const void *)n_new,
                          (const void *)share, (const void *)out, (const void *)lse_out})
        if (!aligned16(x)) return RS_INVALID_ARG;
    const PagedLayout x = paged_layout(s, T_new);
    if (!ws || !aligned16(ws) || ws_bytes < x.total) return RS_WORKSPACE_TOO_SMALL;
    PagedParams a;
    a.q = q, a.k = k_pool, a.v = v_pool;
    a.table = table, a.len = len, a.seq = seq, a.n_new = n_new;
    a.share = x.rows > 0 ? share : nullptr;
    a.out = out, a.lse = lse_out;
    a.cut_o = (float *)((char *)ws + RS_WS_CTRL_BYTES), a.row_o = a.cut_o + x.cut * s->D;
    a.cut_ml = (float *)((char *)ws + x.off_ml), a.row_ml = a.cut_ml + x.cut * 2;
    a.plan = (char *)ws + x.off_plan;
    a.B = s->B, a.Hq = s->Hq, a.Hkv = s->Hkv, a.G = s->Hq / s->Hkv;
    a.S = p->S, a.M = p->M, a.N = p->N, a.shift = __builtin_ctz((unsigned)p->P), a.T = T_new, a.groups = kPagedGroups;
    a.own_rows = many_rows(s, (long)T_new * a.G) ? kMany : kFew;
    a.cut_rows = (int)(x.cut / (2 * kPagedGroups));
    a.scale = scale;
    if (s->dtype == RS_BF16) {
        if (s->D == 128) paged_launch<bf16, 128>(a, (hipStream_t)stream);
        else paged_launch<bf16, 64>(a, (hipStream_t)stream);
    } else {
        if (s->D == 128) paged_launch<float, 128>(a, (hipStream_t)stream);
        else paged_launch<float, 64>(a, (hipStream_t)stream);
    }
    return launch_status();
}

}  // extern "C"
