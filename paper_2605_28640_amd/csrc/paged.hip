// Dense attention of the newest tokens of many sequences over a pool of pages, the pages that neighbours of the list have in
// common read once for all of them (Eq. 4 with every token).
//
// Mathematics.  With z_j = scale q . k_j and any split of the positions into parts, each part leaves m = max z_j, l = sum e^(z_j - m),
// o = sum e^(z_j - m) v_j, and parts join by m = max m_i, (l, o) = sum e^(m_i - m) (l_i, o_i): the shared pages are one
// part, attended by the rows of all sequences of the run at once, a sequence's own pages another, and each is split
// further along its keys for balance.
//
// Two kinds of tile:
//   few rows (at most 32: a sequence's heads at decode; and all of float32): bound by the bytes of K and V.  A wave by itself: it streams
//     32 keys (float32: 16) a step, K from memory into registers in the matrix operand's own layout, V through two LDS tiles of its
//     own, the next step's K and the V of two steps on their way.  No barrier anywhere; what a wave waits for at
//     a tile's beginning and end, the others of its CU fill.
//   many rows (tiles of 128; bfloat16): bound by the matrix units.  A workgroup: every wave takes 32 rows, all four go through the same
//     keys, K and V tiles in a ring of LDS slots, one barrier a step.  Where a sequence's own rows fill more than a small tile, all tiles of
//     the call are of this kind, and a kernel with nothing else in it takes three workgroups to a CU (168 registers, three
//     slots of 16 KB filled two steps ahead) instead of two (four slots, three steps): when it was chosen, eight prompts' questions of 150 to 384 tokens
//     after 16384, 32 heads over 8, 670 us against 731; one prompt of 32768 tokens 9.5 ms against 10.6.
// In both S^T = K Q^T and O^T = V^T P^T, so that a lane holds the keys of one query and P^T goes from the accumulators into the
// second product as it is.
//
// Work.  The tiles of each kind, cut into units of keys, form a line: of every segment (a run's shared pages, a sequence's own) its
// tiles, per KV head.  The workgroups are divided between the kinds by the bytes of their keys, side by side on the CUs; every wave takes an
// equal share of the line of few-row tiles, every workgroup one of the line of many-row tiles, whatever the lengths are.  Where a line is cut follows from the
// lengths alone: each workgroup works it out for itself, by a prefix sum over the list, so lengths live on the device and nothing has to
// be planned by the host.  What a share holds of a tile goes to one of its two boundary records if the tile goes on in another
// share, to the row's record if the row has a second part (shared and own), else straight to the output; a second launch joins the records.
//
// Measured, us back to back on a card at work (bfloat16, 32 heads over 8, D 128, pages of 16 unless said; the bytes of K and V that a call cannot
// do without; by counters, what came from beyond the L2 caches):
//   24 sequences of 40 to 9000 tokens: 82, of which the first launch 76 for 446 MB (449 fetched, 5.9 TB/s)
//   32 sequences that share 32768 tokens and have 30 to 1500 of their own: 65; first launch 56 (237 MB, of which the shared
//     134 MB are met by 128 rows a head; 239 fetched), join 9; 64 that share 4096, 32 heads over 32, pages of 64: 79 (397 MB); 48 in three runs
//     that share 12000, pages of 32: 86.5 (403 MB)
//   8 sequences' 150 to 384 new tokens after 16384: 655 (585 GFLOP, 890 TFLOP/s), join 31 for 100 MB of cut tiles' records; matrix units busy
//     47 % of the cycles at 1.95 to 1.97 GHz, half of the L2's requests miss (2.6 GB fetched for 80 MB of K and V).  From an idle card the first dozen calls take up
//     to 890, the clock not being what it is later
//   one prompt of 4096 tokens 189 to 195 (705 to 727 TFLOP/s), 32768 9300 (946)
//   one sequence of 8000 tokens 21, four of 2000 19.5; float32, 2 sequences of 600 tokens, 4 heads over 2: 13.5, all of it launches and trips to memory
#include <type_traits>

#include "check.h"
#include "common.h"

namespace rs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
constexpr int kPagedGroups = 512;      // two workgroups a CU
constexpr int kManyGroups = 768;       // where all tiles are of many rows: three
constexpr int kCus = 256;
constexpr int kMaxList = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;          // the softmax's reference point moves when the maximum has grown by more (base-2 exponent): weights
                                       // up to 2^8, as exact in float32 and bfloat16 as those up to 1, and the accumulators are rescaled seldom
constexpr int kFew = 32, kMany = 128;  // rows of a tile

// keys a wave of a few-row tile takes at a time
template <typename ST>
constexpr int kKeys = sizeof(ST) == 2 ? 32 : 16;

struct PagedParams {
    const void *q, *k, *v;
    const int32_t *table, *len, *seq, *n_new, *share;
    void *out;
    float *lse;
    float *cut_o, *cut_ml;      // boundary records: [2 shares][rows of a tile] x D, x 2; those of many-row tiles first
    float *row_o, *row_ml;      // row records: [shared, own][B Hq T] x D, x 2
    char *plan;                 // the first workgroup's plan, for the join
    struct JoinEntry *entries;  // [B][Hkv], for the join where a sequence's rows are one tile, else nullptr
    long few_base;              // the first row of the few-row tiles' boundary records
    int few_rows;               // rows that a few-row tile of this call can have
    int own_many;               // whether a sequence's own tiles are of many rows (then all are)
    int groups;                 // workgroups of the first launch
    int B, Hq, Hkv, G, S, M, N, shift, T;
    float scale;
};

struct Seq {
    int L, n, c, first;  // tokens, new ones, pages of the run's shared part (0: none), the run's first place in the list
};
struct Plan {
    Seq *seq;       // [B]
    int *start[2];  // [B + 1] places of the line (of few-row tiles, of many-row tiles) before this entry of the list
    int *members;   // [B] members of the run that begins here (0: none begins, or it shares nothing)
    int *fewest;    // [B] pages a run can share
    int *row;       // [B] the sequence's row of the table
    __device__ __forceinline__ Plan(char *at, int B) : seq((Seq *)at)
    {
        start[0] = (int *)(seq + B);
        start[1] = start[0] + B + 1;
        members = start[1] + B + 1;
        fewest = members + B;
        row = fewest + B;
    }
};
static size_t plan_bytes(int B) { return (size_t)B * 16 + (size_t)(5 * B + 2) * 4; }
constexpr size_t plan_room(int B) { return ((size_t)B * 16 + (size_t)(5 * B + 2) * 4 + 255) & ~(size_t)255; }
constexpr int kPlanShares = 256;  // bytes before the plan in the workspace: how both lines are divided

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long scalar(long x)
{
    return (long)((uint64_t)(uint32_t)scalar((int)(x >> 32)) << 32 | (uint32_t)scalar((int)x));
}
__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }

// What the two kinds of tile differ in; a value, and not a template's argument, so that there is one way through the code for both (more code
// than the 64 KB of the CUs' instruction caches costs every launch the fetching of it).
struct Kind {
    bool many;
    int rows, unit;  // log2 of a tile's rows, of a unit's keys
    // what beginning and ending a tile costs, in units; 32768 shared by 32, 4096 by 64, in us: many-row tiles 1 / 2 / 3 units 61.4, 61.6, 61.7 and
    // 77.5, 78.2, 78.4; few-row 2 / 3 / 4 62.3, 61.6, 61.7 and 78.2 each
    int before;
    // a tile of n units takes n places of its line and those before them; a tile without units none
    __device__ __forceinline__ int places(int n) const { return n > 0 ? n + before : 0; }
    __device__ __forceinline__ int tiles(int r) const { return (int)(((unsigned)r + (1u << rows) - 1) >> rows); }
    __device__ __forceinline__ int units(int keys) const { return (int)(((unsigned)keys + (1u << unit) - 1) >> unit); }
};
template <typename ST>
__device__ __forceinline__ Kind kind_of(bool many)
{
    if (sizeof(ST) == 2 && many) return Kind{true, __builtin_ctz(kMany), 7, 2};
    return Kind{false, __builtin_ctz(kFew), __builtin_ctz(kKeys<ST>), 3};
}

template <typename ST>
__device__ __forceinline__ bool shared_is_many(int rows)
{
    return sizeof(ST) == 2 && rows > kFew;
}

// units of row tile rt of sequence x over its own pages: the keys from the shared ones to the tile's last row
__device__ __forceinline__ int own_units(const Kind &kind, const Seq &x, int rt, int G, int shift, int &k0, int &k1)
{
    const int t0 = (rt << kind.rows) / G, t1 = min(x.n - 1, ((rt << kind.rows) + (1 << kind.rows) - 1) / G);
    k0 = x.c << shift;
    k1 = x.L - x.n + t1 + 1;
    return (t0 >= x.n || k1 <= k0) ? 0 : kind.units(k1 - k0);
}
// places of a sequence's own row tiles rt, rt + step, ...
__device__ __forceinline__ int own_places(const PagedParams &a, const Kind &kind, const Seq &x, int rt, int step)
{
    int sum = 0, k0, k1;
    for (; rt < kind.tiles(x.n * a.G); rt += step) sum += kind.places(own_units(kind, x, rt, a.G, a.shift, k0, k1));
    return sum;
}

// Fills the plan; called by the whole workgroup.
template <typename ST>
__device__ __forceinline__ void make_plan(const PagedParams &a, const Plan &pl)
{
    const int tid = threadIdx.x;
    for (int b = tid; b < a.B; b += kPagedThreads) {
        // (two trips to memory: the list's entries, then length and the run's entry side by side)
        const int s = a.seq[b], f = a.share ? a.share[3 * b] : -1;
        int n = a.n_new ? a.n_new[b] : a.T;
        const int *run = a.share + 3 * (f >= 0 && f <= b ? f : b);
        const int begins = a.share ? run[0] : 0, cnt = a.share ? run[1] : 0, shared = a.share ? run[2] : 0;
        int L = (s >= 0 && s < a.S) ? a.len[s] : 0;
        L = L < 0 ? 0 : min(L, a.M << a.shift);
        n = n < 0 ? 0 : min(n, a.T);
        int first = b, c = 0;
        if (f >= 0 && f <= b && begins == f && cnt > b - f && cnt <= a.B - f && cnt > 1) {
            first = f;
            c = min(max(shared, 0), max(L - n, 0) >> a.shift);
        }
        pl.seq[b] = Seq{L, n, c, first};
        pl.members[b] = (c > 0 && first == b) ? cnt : 0;
        pl.fewest[b] = 0x7fffffff;
        pl.row[b] = s;
    }
    __syncthreads();
    if (a.share) {
        for (int b = tid; b < a.B; b += kPagedThreads) atomicMin(&pl.fewest[pl.seq[b].first], pl.seq[b].c);
        __syncthreads();
    }
    // (a thread's stretch of the list, so that a second pass can add what precedes it)
    __shared__ int tot[2][kPagedWaves];
    const int each = div_up(a.B, kPagedThreads), lo = min(tid * each, a.B), hi = min(lo + each, a.B);
    int sum[2] = {0, 0}, inc[2];
    auto settled = [&](int b) __attribute__((always_inline)) -> Seq {  // with the pages its run shares
        Seq x = pl.seq[b];
        x.c = pl.members[x.first] ? pl.fewest[x.first] : 0;  // (nobody writes members, fewest or first here)
        return x;
    };
    // entries of many tiles: a wave each (a prompt of 32768 tokens has 1024 and more)
    const Kind own_kind = kind_of<ST>(a.own_many);
    const bool by_wave = a.T * a.G > 8 * kFew;
    if (by_wave) {
        for (int b = tid >> 6; b < a.B; b += kPagedWaves) {
            const Seq x = settled(b);
            int own = own_places(a, own_kind, x, lane_id(), kWave);
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) own += __shfl_xor(own, d, kWave);
            if (lane_id() == 0) pl.start[0][b] = own;
        }
        __syncthreads();
    }
    for (int b = lo; b < hi; ++b) {
        const Seq x = settled(b);
        const int own = by_wave ? pl.start[0][b] : own_places(a, own_kind, x, 0, 1);
        int few = a.own_many ? 0 : own, many = a.own_many ? own : 0;
        const int rows = x.c > 0 ? pl.members[b] * a.T * a.G : 0;  // of the run that begins here
        if (rows > 0) {
            const Kind run = kind_of<ST>(shared_is_many<ST>(rows));
            const int more = run.tiles(rows) * run.places(run.units(x.c << a.shift));
            if (run.many) many += more;
            else few += more;
        }
        pl.seq[b].c = x.c;
        pl.start[0][b] = few;
        pl.start[1][b] = many;
        sum[0] += few;
        sum[1] += many;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        inc[k] = wave_scan_i(sum[k]);
        if (lane_id() == kWave - 1) tot[k][tid >> 6] = inc[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int at = inc[k] - sum[k];
        for (int w = 0; w < (tid >> 6); ++w) at += tot[k][w];
        for (int b = lo; b < hi; ++b) {
            const int u = pl.start[k][b];
            pl.start[k][b] = at;
            at += u;
        }
        if (hi == a.B && lo < hi) pl.start[k][a.B] = at;
    }
    __syncthreads();
}

// How many of the workgroups take many-row tiles: by the bytes of both kinds' keys, a multiple of the eight XCDs, at least eight for
// each kind that there is.  A unit of many-row tiles is 128 keys, one of few-row tiles 32; a byte of it is weighted 1.3 for the arithmetic (units
// weighted 5 / 5.25 / 5.5: 32768 tokens shared by 32 sequences 61 us each, 4096 by 64, 32 heads of 64, 60.8 / 54.0 / 54.0, 12000 in three runs
// 80.7 / 80.5 / 83.5).  An even number to an XCD, whose two halves then lie alike, the first on CUs by themselves, the second beside the first:
// odd numbers leave CUs with one of each kind.  38 / 39 / 40 / 41 of 64, 32768 tokens by 32: 61.3 / 65.3 / 61.5 / 63.7; 30 / 31 / 32 / 33, 16384 by 16
// 42.0 / 47.1 / 42.7 / 47.8; 17 / 18 / 19 / 20, 8192 by 9 with 2000 to 4000 of their own 45.4 / 42.3 / 45.2 / 43.0; 11 / 12, 4096 by 64, 32 heads, 83.3 / 78.0.
__device__ __forceinline__ int many_groups(int few_line, int many_line, int groups)
{
    if (many_line == 0 || few_line == 0) return many_line > 0 ? groups : 0;
    const float many = (float)many_line * 5.25f, part = many / (many + (float)few_line);  // (in bfloat16's units: both kinds exist only there)
    return 8 * max(1, min(kPagedGroups / 8 - 1, 2 * (int)(part * (kPagedGroups / 16) + 0.5f)));
}
// A line's division into shares.  With few places, equal ones, of at least a 24th of what an entry of the list has (1 to 8 places; a sixth of many rows', whose
// records are four times as large: a 24th / 12th / sixth / third, 32 heads over 8, 64 tokens each after 600 to 900 52.3 / 52.2 / 45.8 / 47.7, 19 each
// after 1376 shared ones 35.1 / 35.1 / 35.3 / 32.3): a share more
// is a record more for the join (at least 1 / 2 / 4 / 8 places, us: one sequence of 8000 tokens 44.5 / 28.5 / 22.0 / 21.1, of 32000
// 62.8 / 62.8 / 58.8 / 43.8, four of 2000 24.4 / 19.8 / 18.2 / 19.3, eight of 2000 to 3000 with 4 new tokens each 32.5 / 32.5 / 29.2 / 27.0, two of 600, 4 heads
// over 2, 13.4 / 13.3 / 13.9 / 17.5; 24 new tokens each after 600 to 900, 16 heads over 8, float32, 62.3 / 62.1 / 50.9 / 58.1).  Else shares by the eight
// XCDs, in each those of its first 32 workgroups 11 places for every 9 of the others': two workgroups are on a CU, and the one that came first is served
// first by its memory path (four sequences of 65536 tokens, 8 heads, with equal shares: every one of the first 256 workgroups done after
// 131-145 us, every other after 157-171).  10:10 / 11:9 / 12:8, us: 32768 shared by 32 60.3 / 61.6 / 63.6, 4096 by 64 78.4 / 78.2 / 78.5,
// 12000 in three runs 80.0 / 78.5 / 78.3, 24 of 40 to 3000, 32 heads, 107.0 / 105.2 / 105.2.  Where there are three to a CU, 12 for 9 (questions after
// 16384, 9:9 / 11:9 / 12:9 / 13:9: 663 / 662 / 647 / 662).
struct Shares {
    static constexpr int kOlder = 11, kOldest = 12, kNewer = 9;
    int line, n;             // places of a KV head, shares
    int of_xcd, older, weight;  // shares of an XCD, those of its first workgroups, the weight of one of these
    int sum;                 // the weights of an XCD's shares together (0: equal shares)
    int each, more;          // equal shares: the first `more` have each + 1
    long all;
    double unit;             // places for each unit of weight
    // reciprocals: a division of integers, or one in 64 bits, costs the beginning of every launch as much as 30 other instructions
    float per_unit;          // of unit
    float per_xcd, per_sum;  // of of_xcd, of sum; equal shares: of each, of each + 1
    Shares() = default;
    __device__ __forceinline__ Shares(const Plan &pl, int B, int Hkv, int all_groups, bool MANY)
    {
        static_assert(sizeof(Shares) <= kPlanShares / 2, "room in the workspace");
        const int f = scalar(pl.start[0][B]), m = scalar(pl.start[1][B]), groups = many_groups(f, m, all_groups);
        line = MANY ? m : f;
        all = (long)line * Hkv;
        const int first = groups == kManyGroups ? kCus / 8 : groups / 16;  // many-row workgroups among an XCD's first 32
        of_xcd = MANY ? groups / 8 : (all_groups - groups) / 8 * kPagedWaves;
        older = MANY ? first : (kCus / 8 - first) * kPagedWaves;
        weight = groups == kManyGroups ? kOldest : kOlder;
        n = 8 * of_xcd;
        sum = 0;
        each = 1, more = 0, unit = 0., per_unit = per_xcd = per_sum = 0.f;
        if (n > 0 && all >= 4l * n) {
            sum = older * weight + (of_xcd - older) * kNewer;
            per_sum = __builtin_amdgcn_rcpf((float)sum);
            per_xcd = __builtin_amdgcn_rcpf((float)of_xcd);
            unit = (double)all * (double)(0.125f * per_sum);  // (off by 2^-22 of it: begin() rounds a whole number back up)
            per_unit = (float)(8 * sum) * __builtin_amdgcn_rcpf((float)all);
        } else {
            const int least = max(1, min(8, (int)((float)line * __builtin_amdgcn_rcpf((MANY ? 6.f : 24.f) * (float)B))));
            n = min(n, quotient((int)all + least - 1, __builtin_amdgcn_rcpf((float)least)));
            if (n > 0) {
                each = (int)all / n;
                more = (int)all - each * n;
                per_xcd = __builtin_amdgcn_rcpf((float)each);
                per_sum = __builtin_amdgcn_rcpf((float)(each + 1));
            }
        }
    }
    // w / d for small whole numbers, from 1 / d: half a unit away from the next one, which is more than the rounding
    __device__ __forceinline__ static int quotient(int w, float per_d) { return (int)(((float)w + 0.5f) * per_d); }
    __device__ __forceinline__ long begin(int w) const
    {
        if (sum == 0) return w * each + min(w, more);
        if (w >= n) return all;
        const int x = quotient(w, per_xcd), i = w - x * of_xcd;
        return (long)((double)(x * sum + min(i, older) * weight + max(i - older, 0) * kNewer) * unit + 0.0625);
    }
    __device__ __forceinline__ int owner(long place) const
    {
        int w;
        if (sum == 0) {
            const int longer = more * (each + 1), p = (int)place;
            w = p < longer ? quotient(p, per_sum) : more + quotient(p - longer, per_xcd);
        } else {
            const int at = (int)((float)place * per_unit), x = quotient(at, per_sum), r = at - x * sum;
            w = x * of_xcd + (r < older * weight ? (weight == kOldest ? r / kOldest : r / kOlder) : older + (r - older * weight) / kNewer);
        }
        w = max(0, min(w, n - 1));
        while (w > 0 && begin(w) > place) --w;  // (at most a step or two: the quotients are rounded)
        while (w + 1 < n && begin(w + 1) <= place) ++w;
        return w;
    }
};
// where the part of a tile (its units at s0 .. s1 - 1) that lies in [wb, we) goes: 2: all of it is there; 0, 1: a boundary record
__device__ __forceinline__ int record_of(long s0, long s1, long wb, long we) { return (s0 >= wb && s1 <= we) ? 2 : s0 <= wb ? 0 : 1; }
// the first row of a boundary record
__device__ __forceinline__ long cut_row(const PagedParams &a, bool many, long share, int record)
{
    return many ? (2 * share + record) * kMany : a.few_base + (2 * share + record) * a.few_rows;
}

// one tile of rows over a run of keys
struct TileWork {
    int kvh, b, rt, rows;     // rows: of the segment (the tile takes those from rt * (its kind's rows) on)
    bool shared;
    int row_seq;              // whose table row names the pages
    int key0, units, limit;   // first key, units of keys from there, keys that exist (later ones are nobody's)
    int record;               // record_of()
    long cut;                 // cut_row() of the boundary record
    bool direct;              // a whole tile without a second part
    int entries;              // this lane's first entry of the table (PageList)
};

// the tile that place `at` of the whole line belongs to; its units are those at s0 .. s1 - 1
template <typename ST>
__device__ __forceinline__ void find_tile(const PagedParams &a, const Plan &pl, const Kind &kind, long at, int line, TileWork &w, long &s0, long &s1)
{
    const int *start = pl.start[kind.many];
    w.kvh = (int)(at / line);
    int off = (int)(at % line), n = 0, lo = 0;
    for (int hi = a.B; hi - lo > 1;) {  // the last entry that begins at or before off (entries without places are passed over)
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= off) lo = mid;
        else hi = mid;
    }
    w.b = lo;
    off -= start[lo];
    const Seq x = pl.seq[lo];
    w.row_seq = pl.row[lo];
    w.key0 = 0;
    w.shared = false;
    const int run_rows = x.c > 0 ? pl.members[lo] * a.T * a.G : 0;
    if (run_rows > 0 && shared_is_many<ST>(run_rows) == kind.many) {
        w.rows = run_rows;
        w.limit = x.c << a.shift;
        n = kind.units(w.limit);
        const int su = kind.places(n), st = kind.tiles(w.rows);
        w.shared = off < su * st;
        if (w.shared) {
            w.rt = off / su;
            off -= w.rt * su;
        } else {
            off -= su * st;
        }
    }
    if (!w.shared) {
        w.rows = x.n * a.G;
        for (w.rt = 0;; w.rt += kWave) {  // 64 tiles at a time, one a lane
            int k1, i = 0;
            const int p = kind.places(own_units(kind, x, w.rt + lane_id(), a.G, a.shift, w.key0, k1));
            if (scalar(w.rows) >> kind.rows) {  // which of them
                const int inc = wave_scan_i(p);
                const uint64_t past = __ballot(off < inc);
                i = past ? __builtin_ctzll(past) : kWave - 1;
                off -= __builtin_amdgcn_readlane(past ? inc - p : inc, i);
                if (!past) continue;
            }
            n = __builtin_amdgcn_readlane(p, i) - kind.before;
            w.limit = __builtin_amdgcn_readlane(k1, i);
            w.rt += i;
            break;
        }
    }
    s0 = scalar(at - off + kind.before);
    s1 = s0 + scalar(n);
    // (what is read from LDS is the same for all lanes, which the compiler does not know: as vectors these would take the
    // registers of the accumulators)
    w.kvh = scalar(w.kvh), w.b = scalar(w.b), w.rt = scalar(w.rt), w.rows = scalar(w.rows), w.row_seq = scalar(w.row_seq);
    w.key0 = scalar(w.key0), w.limit = scalar(w.limit);
    w.shared = scalar(w.shared) != 0;
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
    const Seq x = pl.seq[bq];
    return t < x.n && (!w.shared || x.first == w.b);  // (of runs that overlap, an entry belongs to the one that it names)
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
    const long at = whole ? (w.shared ? 0 : (long)a.B * a.Hq * a.T) + row : w.cut + r;
    *reinterpret_cast<f32x4 *>((whole ? a.row_o : a.cut_o) + at * D + c) = o;
    if (c == 0) *reinterpret_cast<float2 *>((whole ? a.row_ml : a.cut_ml) + at * 2) = make_float2(m, l);
}

// ---- pages -----------------------------------------------------------------------------------------------------
// Which rows hold the keys from `first` on, 16 at a time (a page is 16 keys and more).  64 entries of the table at a time, one a lane.
struct PageList {
    const int32_t *row;
    int first, last, limit, N, shift, listed;  // last: groups of 16 that are asked for
    // this lane's entry of the 64 from n on, as the table has it
    __device__ __forceinline__ int fetch(int n) const
    {
        const int m = n + lane_id(), k = first + 16 * m;
        int page = -1;
        if (m < last && k < limit) page = row[k >> shift];
        return page;
    }
    __device__ __forceinline__ void take(int page)
    {
        listed = (page < 0 || page >= N) ? -1 : page;
        asm volatile("" : "+v"(listed));  // (waited for here, and not by every step)
    }
    // rows that exist (0 .. 16) of group n, and the first of them; asked for in ascending order by the whole wave
    __device__ __forceinline__ int rows(int n, long &at)
    {
        if ((n & 63) == 0 && n > 0) take(fetch(n));
        const int page = __builtin_amdgcn_readlane(listed, n & 63), k = first + 16 * n, left = limit - k;
        at = page < 0 ? 0l : ((long)page << shift) + (k & ((1 << shift) - 1));
        // (a scalar, which the compiler does not see in the clamp: the descriptors made of it would be a loop over the lanes each)
        return __builtin_amdgcn_readfirstlane(page < 0 || left < 0 ? 0 : left < 16 ? left : 16);
    }
};
template <typename ST>
__device__ __forceinline__ PageList page_list(const PagedParams &a, const Kind &kind, const TileWork &w)
{
    constexpr int STEP = kKeys<ST>;  // (of both kinds)
    const int end = min(w.limit, w.key0 + (w.units << kind.unit));
    return PageList{a.table + (long)w.row_seq * a.M, w.key0, (end - w.key0 + STEP - 1) / STEP * (STEP / 16), w.limit, a.N, a.shift, -1};
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

// the LDS of a workgroup: eight tiles of 32 bfloat16 (16 float32) rows
struct Ring {
    char *k0, *k1, *k2, *k3, *v0, *v1, *v2, *v3;
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
// a matrix product would take 0 times it.  D / 4 lanes a row, of the wave (few rows) or the workgroup.
template <typename ST, int D>
__device__ __forceinline__ void attend_by_key(const PagedParams &a, const Plan &pl, const Kind &kind, const TileWork &w)
{
    constexpr int C4 = D / 4;
    const int c4 = threadIdx.x % C4, end = min(w.limit, w.key0 + (w.units << kind.unit)), n_rows = 1 << kind.rows;
    const int grp = (kind.many ? threadIdx.x : lane_id()) / C4, groups = (kind.many ? kPagedThreads : kWave) / C4;
    const int32_t *pages = a.table + (long)w.row_seq * a.M;
    const long pool = (long)w.kvh * ((long)a.N << a.shift);
    const float cs = a.scale * kLog2e;
#pragma unroll 1
    for (int r = grp; r < n_rows; r += groups) {
        int bq, t, g;
        if (!query_of(a, pl, w, (w.rt << kind.rows) + r, bq, t, g)) continue;
        const long row = out_row(a, w, bq, t, g);
        const int last = w.shared ? end - 1 : min(end - 1, pl.seq[bq].L - pl.seq[bq].n + t);
        float q[4], m = -INFINITY, l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = to_f32(((const ST *)a.q)[row * D + 4 * c4 + j]);
#pragma unroll 1
        for (int key = w.key0; key <= last; ++key) {
            const int page = pages[key >> a.shift];
            if (page < 0 || page >= a.N) continue;
            const long at = (pool + ((long)page << a.shift) + (key & ((1 << a.shift) - 1))) * D + 4 * c4;
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) z = fmaf(q[j], to_f32(((const ST *)a.k)[at + j]), z);
            z = group_sum<C4>(z) * cs;
            const float top = fmaxf(m, z), bias = top == -INFINITY ? 0.f : top;  // (infinities as the products' way has them)
            const float f = __builtin_amdgcn_exp2f(m - bias), p = __builtin_amdgcn_exp2f(z - bias);
            m = top;
            l = l * f + p;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = o[j] * f + p * to_f32(((const ST *)a.v)[at + j]);
        }
        put4<ST, D>(a, w, row, r, 4 * c4, o, m, l);
    }
}

// ---- few rows --------------------------------------------------------------------------------------------------
// 16-wide matrix instructions: lane (l16, lg) = (lane % 16, lane / 16) holds query l16 and, of every 16 keys, 4 lg .. 4 lg + 3.
// K operand: row l16, 16 bytes at chunk 4 kk + lg, straight from memory (a load touches 64 bytes of each of 16 rows; the lines
// are used up by the loads beside it: streaming 446 MB so, 5.9 TB/s).  V operand, bfloat16: transpose reads of the row-major tile, chunks of a row
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
__device__ __forceinline__ void attend_few(const PagedParams &a, const Plan &pl, const TileWork &w, char *const even, char *const odd_tile)
{
    using Rows = FewRows<ST, D>;
    constexpr bool BF = sizeof(ST) == 2;
    constexpr int KT = kKeys<ST>, NH = KT / 16, ROW = Rows::ROW;
    constexpr int NDT = D / 16, NK = BF ? D / 32 : D / 16;  // 16-channel tiles of O^T; 16-byte operands of a row
    const int lane = lane_id(), l16 = lane & 15, lg = lane >> 4;

    const long pool = (long)w.kvh * ((long)a.N << a.shift);
    const ST *kb = (const ST *)a.k + pool * D, *vb = (const ST *)a.v + pool * D;
    PageList pages = page_list<ST>(a, kind_of<ST>(false), w);
    pages.take(w.entries);

    f32x4 kf[NH][NK];
    struct Where {
        long at[NH];
        int valid[NH];
    };
    const uint32_t k_at = (uint32_t)(l16 * ROW + lg * 16);
    auto look_up = [&](int u) __attribute__((always_inline)) -> Where {  // (past the last step: no rows)
        Where x;
#pragma unroll
        for (int h = 0; h < NH; ++h) x.valid[h] = pages.rows(u * NH + h, x.at[h]);
        return x;
    };
    auto load_k = [&](const Where &x) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const LdsSource src = lds_source_sized(kb + x.at[h] * D, x.valid[h] * ROW);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) kf[h][kk] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(src, k_at + 64 * kk, 0, 2));
        }
        pin();
    };
    auto load_v = [&](const Where &x, char *tile) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < NH; ++h) Rows::load_v(lds_source_sized(vb + x.at[h] * D, x.valid[h] * ROW), tile + h * 16 * ROW);
        pin();
    };
    // V of a step is always on its way before its K, so that K being there means V is
    Where x0 = look_up(0);
    load_v(x0, even);
    load_k(x0);
    Where x1 = look_up(1);
    load_v(x1, odd_tile);

    // ---- this lane's queries ----
    f32x4 qf[RT][NK];
    bool real[RT];
    long row[RT];
    int last[RT];                 // the last position the row sees (-1: there is no such row)
    int first_last = 0x7fffffff;  // the smallest of the tile's rows (what comes of rows that do not exist is dropped)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        int bq, t, g;
        real[rt] = query_of(a, pl, w, w.rt * kFew + rt * 16 + l16, bq, t, g);
        last[rt] = -1;
        row[rt] = 0;
        if (real[rt]) {
            row[rt] = out_row(a, w, bq, t, g);
            last[rt] = pl.seq[bq].L - pl.seq[bq].n + t;
        }
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const char *>((const ST *)a.q + row[rt] * D) + 64 * kk + 16 * lg);
            qf[rt][kk] = real[rt] ? x : f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (real[rt]) first_last = min(first_last, last[rt]);
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) first_last = min(first_last, __shfl_xor(first_last, m, kWave));
    first_last = __builtin_amdgcn_readfirstlane(first_last);
    if (w.shared || first_last >= w.limit - 1) first_last = 0x7fffffff;  // every row sees all keys there are

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
        const int r = 4 * lg + (l16 >> 2);
        v_at[0] = (uint32_t)(r * ROW + ((((l16 & 3) >> 1) ^ Rows::v_swizzle(r)) * 16) + 8 * (l16 & 1));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v_at[j] = (uint32_t)((4 * lg + j) * ROW + (((l16 >> 2) ^ Rows::v_swizzle(4 * lg + j)) * 16) + 4 * (l16 & 3));
    }

    bool odd = false;  // values that are not finite where some row may not look
    const int n_steps = pages.last / NH;
#pragma unroll 1
    for (int u = 0; u < n_steps; ++u) {
        const int key = w.key0 + u * KT;
        char *const cV = (u & 1) ? odd_tile : even;
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
        load_k(x1);
        // ---- softmax, base 2 ----
        const bool edge = key + KT - 1 > first_last;  // some row does not see some key of this step
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int h = 0; h < NH; ++h) s[rt][h] *= cs;
        if (edge || x0.valid[0] < 16 || x0.valid[NH - 1] < 16) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int h = 0; h < NH; ++h) {
                    const int sees = min(x0.valid[h], edge ? last[rt] + 1 - key - 16 * h : 16) - 4 * lg;  // of the lane's four
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
        // ---- O^T += V^T P^T (weights rounded to the storage type: half a step of 2^-8 of each, of which a row has many) ----
        pin();
        wait_loads<NH *(NK + Rows::NL)>();  // V is here (the next V and the next K may be on their way)
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
        x0 = x1;
        x1 = look_up(u + 2);
        load_v(x1, cV);
    }
    wait_loads<0>();  // (nothing lands in this LDS any more)
    if (__any(odd)) return attend_by_key<ST, D>(a, pl, kind_of<ST>(false), w);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float sum = quad_sum(l[rt]);
        if (real[rt]) {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) put4<ST, D>(a, w, row[rt], rt * 16 + l16, 16 * dt + 4 * lg, oacc[rt][dt], m[rt], sum);
        }
    }
}

// ---- many rows -------------------------------------------------------------------------------------------------
// 32-wide matrix instructions: lane (lq, h) = (lane % 32, lane / 32) holds query lq and keys 8 i + 4 h .. + 3 of a step's 32.  With three slots
// (three waves to a SIMD) registers are what is short: no step is passed over (one that no row of the wave sees comes out as nothing,
// its weights are 0 and its values finite, or the tile is taken key by key), since a way round the arithmetic keeps a second set of accumulators,
// and what a lane's addresses differ in is worked out anew every step.
template <int D, int SLOTS>
__device__ __forceinline__ void attend_many(const PagedParams &a, const Plan &pl, const TileWork &w, const Ring &lds)
{
    constexpr int NC = D / 16, NDT = D / 32, CR = D / 8, RW = 64 / CR, RPI = kPagedWaves * RW, CPT = 32 / RPI, ROW = 2 * D;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lq = lane & 31, h = lane >> 5;
    const long pool = (long)w.kvh * ((long)a.N << a.shift);
    const bf16 *kb = (const bf16 *)a.k + pool * D, *vb = (const bf16 *)a.v + pool * D;
    PageList pages = page_list<bf16>(a, kind_of<bf16>(true), w);
    const int n_steps = pages.last / 2;
    pages.take(w.entries);

    // staging: pass i of a tile: this wave fetches RW rows, rows RPI i + RW wave on, all of one 16-key group
    const int row0 = (RW * wave + lane / CR) & 15;  // in the group
    const uint32_t gk = (uint32_t)(row0 * ROW + (((lane % CR) ^ chunk_swizzle<D>(row0)) * 16));
    const uint32_t gv = (uint32_t)(row0 * ROW + (((lane % CR) ^ chunk_swizzle<D>(row0 & 7)) * 16));
    LdsSource k_src[CPT], v_src[CPT];
    auto look_up = [&](int step) __attribute__((always_inline)) -> int {  // valid rows of the two groups, 8 bits each
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
    int valid2 = 0;
    if constexpr (SLOTS == 4) {
        valid2 = look_up(2);
#pragma unroll
        for (int i = 0; i < CPT; ++i) stage_k(i, lds.k2), stage_v(i, lds.v2);
    }

    // ---- this lane's query ----
    int bq = 0, t = 0, g = 0;
    const int r = wave * 32 + lq;
    const bool real = query_of(a, pl, w, w.rt * kMany + r, bq, t, g);
    const long row = real ? out_row(a, w, bq, t, g) : 0;
    const int last = real ? pl.seq[bq].L - pl.seq[bq].n + t : -1;
    bf16x8 qf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>((const bf16 *)a.q + row * D + 16 * c + 8 * h);
        qf[c] = __builtin_bit_cast(bf16x8, real ? x : f32x4{0.f, 0.f, 0.f, 0.f});
    }
    int first_last = real ? last : 0x7fffffff, wave_last = last;  // the smallest and the largest of the wave's rows
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        first_last = min(first_last, __shfl_xor(first_last, x, kWave));
        wave_last = max(wave_last, __shfl_xor(wave_last, x, kWave));
    }
    first_last = __builtin_amdgcn_readfirstlane(first_last);
    wave_last = __builtin_amdgcn_readfirstlane(wave_last);
    if (w.shared) first_last = 0x7fffffff, wave_last = wave_last >= 0 ? 0x7fffffff : -1;
    // the smallest of the tile's rows (later positions are later rows of it); as far as there are keys that it does not see
    int tile_first = pl.seq[w.b].L - pl.seq[w.b].n + w.rt * kMany / a.G;
    if (w.shared || tile_first >= w.limit - 1) tile_first = 0x7fffffff;
    bool odd = false;  // values that are not finite where some row may not look

    // operand addresses inside a tile: K row lq, chunk 2 c + h; V through the transpose read, lane = 32 h + 16 dg + L supplying 8 bytes of row
    // 16 c + 4 h + L / 4 (+ 8 for the second read) at channel 32 dt + 16 dg + 4 (L % 4)
    const int L16 = lane & 15, dg = (lane >> 4) & 1;
    uint32_t koff = (uint32_t)(lq * ROW + ((h ^ chunk_swizzle<D>(lq)) * 16));
    const int rowa = 4 * h + (L16 >> 2);
    uint32_t voff = (uint32_t)(rowa * ROW + (((2 * dg + ((L16 & 3) >> 1)) ^ chunk_swizzle<D>(rowa)) * 16) + 8 * (L16 & 1));

    f32x16 oacc[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] = 0.f;
    const float cs = __int_as_float(scalar(__float_as_int(a.scale * kLog2e)));
    float m = -INFINITY, l = 0.f;
    wait_loads<2 * (SLOTS - 2) * CPT>();  // the first tile has landed
    asm volatile("s_barrier" ::: "memory");

    auto step = [&](auto buf_tag, int it) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_tag)::value;
        const char *cK = BUF == 0 ? lds.k0 : BUF == 1 ? lds.k1 : BUF == 2 ? lds.k2 : lds.k3, *cV = BUF == 0 ? lds.v0 : BUF == 1 ? lds.v1 : BUF == 2 ? lds.v2 : lds.v3;
        asm volatile("" : "+v"(koff), "+v"(voff));  // (else the 12 addresses made of them are kept in registers)
        constexpr int TO = (BUF + SLOTS - 1) % SLOTS;  // what the step before this one has read
        char *nK = TO == 0 ? lds.k0 : TO == 1 ? lds.k1 : TO == 2 ? lds.k2 : lds.k3, *nV = TO == 0 ? lds.v0 : TO == 1 ? lds.v1 : TO == 2 ? lds.v2 : lds.v3;
        const int key = w.key0 + it * 32, here = valid0;
        const int then = look_up(it + SLOTS - 1);  // (past the last step: descriptors of no rows)
        valid0 = valid1;
        valid1 = SLOTS == 4 ? valid2 : then;
        valid2 = then;
        const bool live = SLOTS == 3 || (key <= wave_last && it < n_steps);
        if (key + 31 > tile_first) odd |= not_finite<bf16>(cV, threadIdx.x, kPagedThreads, 32 * ROW / 16);
        if (!live) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) stage_k(i, nK), stage_v(i, nV);
        }
        if (live) {
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
            asm volatile("" : "+v"(s));  // (nothing of what follows is begun before this: it would not fit beside the scores)
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
        // the next step's tile has landed (those after it may be on their way), and this wave has read what it needs
        __builtin_amdgcn_s_waitcnt(0x0070 | (2 * (SLOTS - 2) * CPT));
        asm volatile("s_barrier" ::: "memory");
    };
    // (whole turns of the ring: steps past the last one only pass the barrier.  With ways out between the steps the compiler keeps two
    // sets of accumulators and copies one to the other every step.)
#pragma unroll 1
    for (int it = 0; it < n_steps; it += SLOTS) {
        step(std::integral_constant<int, 0>{}, it);
        step(std::integral_constant<int, 1>{}, it + 1);
        step(std::integral_constant<int, 2>{}, it + 2);
        if constexpr (SLOTS == 4) step(std::integral_constant<int, 3>{}, it + 3);
    }
    wait_loads<0>();  // (nothing lands in the ring any more)
    if (__syncthreads_or(odd)) return attend_by_key<bf16, D>(a, pl, kind_of<bf16>(true), w);
    const float sum = half_pair_sum(l);
    int again = threadIdx.x;  // (the row is found again: kept through the loop it would take more registers than there are)
    asm volatile("" : "+v"(again));
    const int r_out = wave * 32 + (again & 31);
    if (query_of(a, pl, w, w.rt * kMany + r_out, bq, t, g)) {
        const long row_out = out_row(a, w, bq, t, g);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = oacc[dt][4 * i + j];
                put4<bf16, D>(a, w, row_out, r_out, 32 * dt + 8 * i + 4 * h, o, m, sum);
            }
    }
}

// The shares that a tile's records come from: w0 .. w1 (none: w1 < w0).  One share: the row's record; else boundary records, the second one
// of share w0 where that began before the tile.
struct Span {
    int w0, w1, begun;
};
__device__ __forceinline__ Span span_of(const Shares &sh, long s0, int units)
{
    if (units == 0) return Span{0, -1, 0};
    const int w0 = sh.owner(s0), w1 = s0 + units <= sh.begin(w0 + 1) ? w0 : sh.owner(s0 + units - 1);
    return Span{w0, w1, s0 > sh.begin(w0) ? 1 : 0};
}
// What the join of the rows of a list's entry and KV head goes by, where they are one tile of their own.  Worked out by a wave of each of the
// first launch's workgroups, so that the second launch has nothing to do but to fetch.
struct JoinEntry {
    Span own, shared[2];  // of the own tile; of the run's tiles that hold the entry's rows (they may go on in a second one)
    int n, row0, many;    // new tokens; the first row in the run's tile; whether that is of many rows
};
// a part of the entry: 0: its own tile and the numbers, 1, 2: the run's tiles (a thread each: the divisions take their time).  One way
// through for all of them and both kinds: as a way each this was a quarter of the kernel's code, more than the CUs' instruction
// caches hold (64 KB), which every launch began by fetching.
template <typename ST>
__device__ __forceinline__ void fill_join_entry(const PagedParams &a, const Plan &pl, const Shares &few, const Shares &many, int b, int kvh,
                                                int part, JoinEntry &e)
{
    const Seq x = pl.seq[b];
    const bool own = part == 0;
    const int head = own ? b : x.first, run_rows = x.c > 0 ? pl.members[head] * a.T * a.G : 0;  // (0 too: no run begins at b)
    const Kind run = kind_of<ST>(shared_is_many<ST>(run_rows)), kind = own ? kind_of<ST>(a.own_many) : run;
    const int row = (b - x.first) * a.T * a.G, run_units = run.units(x.c << a.shift);
    int units, tile, k0, k1;  // of the tile; tiles of the run before it among the entry's places
    if (own) {
        units = own_units(kind, x, 0, a.G, a.shift, k0, k1);
        tile = run.many == kind.many ? run.tiles(run_rows) : 0;
    } else {
        tile = (row >> run.rows) + part - 1;
        units = tile < run.tiles(run_rows) ? run_units : 0;
    }
    const Shares sh = kind.many ? many : few;
    const long s0 = (long)kvh * sh.line + pl.start[kind.many][head] + (long)tile * run.places(run_units) + kind.before;
    const Span span = span_of(sh, s0, units);
    if (own) {
        e.own = span;
        e.n = x.n;
    } else {
        e.shared[part - 1] = span;
        if (part == 1) e.row0 = row & ((1 << run.rows) - 1), e.many = run.many;
    }
}

// ALL_MANY: for calls all of whose tiles are of many rows
template <typename ST, int D, bool ALL_MANY>
__global__ __launch_bounds__(kPagedThreads) __attribute__((amdgpu_waves_per_eu(ALL_MANY ? 3 : 2, ALL_MANY ? 3 : 2))) void paged_attend_kernel(const PagedParams a)
{
    constexpr int TILE = kKeys<ST> * D * (int)sizeof(ST);
    __shared__ __attribute__((aligned(1024))) char k0[TILE];
    __shared__ __attribute__((aligned(1024))) char k1[TILE];
    __shared__ __attribute__((aligned(1024))) char k2[TILE];
    __shared__ __attribute__((aligned(1024))) char v0[TILE];
    __shared__ __attribute__((aligned(1024))) char v1[TILE];
    __shared__ __attribute__((aligned(1024))) char v2[TILE];
    __shared__ __attribute__((aligned(ALL_MANY ? 16 : 1024))) char k3[ALL_MANY ? 16 : TILE];
    __shared__ __attribute__((aligned(ALL_MANY ? 16 : 1024))) char v3[ALL_MANY ? 16 : TILE];
    extern __shared__ __attribute__((aligned(16))) char lds_plan[];
    const Ring ring{k0, k1, k2, k3, v0, v1, v2, v3};
    const Plan pl(lds_plan, a.B);
    make_plan<ST>(a, pl);
    const Shares few(pl, a.B, a.Hkv, a.groups, false), many(pl, a.B, a.Hkv, a.groups, true);
    if (blockIdx.x == 0) {  // for the join
        const Plan to(a.plan + kPlanShares, a.B);
        if (threadIdx.x == 0) {
            *reinterpret_cast<Shares *>(a.plan) = few;
            *reinterpret_cast<Shares *>(a.plan + kPlanShares / 2) = many;
        }
        for (int b = threadIdx.x; b <= a.B; b += kPagedThreads) {
            to.start[0][b] = pl.start[0][b];
            to.start[1][b] = pl.start[1][b];
            if (b == a.B) break;
            to.seq[b] = pl.seq[b];
            to.members[b] = pl.members[b];
            to.row[b] = pl.row[b];
        }
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (a.entries && wave == kPagedWaves - 1) {  // (here, and not when all is done: what it needs would have to be kept in registers until then)
        for (int p = blockIdx.x + a.groups * (lane_id() / 4); p < a.B * a.Hkv; p += a.groups * 16)
            if (lane_id() % 4 < 3) fill_join_entry<ST>(a, pl, few, many, p / a.Hkv, p % a.Hkv, lane_id() % 4, a.entries[p]);
    }
    // Workgroups are dealt to the eight XCDs in turn, and there in turn to the CUs.  On every XCD the two kinds are spread evenly, and
    // those of one XCD take neighbouring shares of a line, tiles of one KV head as a rule, whose rows they find in their L2; less
    // work than workgroups goes to all XCDs.
    const int xcd = blockIdx.x % 8, in_xcd = blockIdx.x / 8, groups = many_groups(scalar(pl.start[0][a.B]), scalar(pl.start[1][a.B]), a.groups), of_xcd = a.groups / 8;
    const int each = groups / 8, before = in_xcd * each / of_xcd;  // many-row workgroups of an XCD, those before this one
    // the next part of a share, with the first entries of its table row on their way
    auto next = [&](const Kind &kind, const Shares &sh, int me, TileWork &w, long &at, long wb, long we) __attribute__((always_inline)) -> bool {
        while (at < we) {
            long s0, s1;
            find_tile<ST>(a, pl, kind, at, sh.line, w, s0, s1);
            const long from = max(at, s0), to = min(we, s1);
            at = s1;
            if (from >= to) continue;  // only places before the units
            w.key0 += (int)(from - s0) << kind.unit;
            w.units = (int)(to - from);
            w.record = record_of(s0, s1, wb, we);
            w.cut = cut_row(a, kind.many, me, w.record & 1);
            w.direct = w.record == 2 && !w.shared && scalar(pl.seq[w.b].c) == 0;
            w.entries = page_list<ST>(a, kind, w).fetch(0);
            return true;
        }
        return false;
    };
    if (ALL_MANY || (in_xcd + 1) * each / of_xcd > before) {
        if constexpr (sizeof(ST) == 2) {
            const Kind kind = kind_of<ST>(true);
            const int me = many.n < groups ? before * 8 + xcd : xcd * each + before;
            if (me >= many.n) return;
            const long wb = many.begin(me), we = many.begin(me + 1);
            long at = wb;
            TileWork w, then;
            bool more = next(kind, many, me, w, at, wb, we);
#pragma unroll 1
            while (more) {
                more = next(kind, many, me, then, at, wb, we);
                attend_many<D, ALL_MANY ? 3 : 4>(a, pl, w, ring);
                w = then;
            }
        }
    } else if constexpr (!ALL_MANY) {
        const Kind kind = kind_of<ST>(false);
        char *const even = wave == 0 ? k0 : wave == 1 ? k2 : wave == 2 ? v0 : v2, *const odd = wave == 0 ? k1 : wave == 1 ? k3 : wave == 2 ? v1 : v3;
        const int mine = in_xcd - before, of = of_xcd - each;  // few-row workgroups of the XCD
        const int me = few.n < of * 8 * kPagedWaves ? (wave * of + mine) * 8 + xcd : (xcd * of + mine) * kPagedWaves + wave;
        if (me >= few.n) return;
        const long wb = few.begin(me), we = few.begin(me + 1);
        long at = wb;
        TileWork w, then;
        bool more = next(kind, few, me, w, at, wb, we);
#pragma unroll 1
        while (more) {
            more = next(kind, few, me, then, at, wb, we);
            if (w.rows - w.rt * kFew <= 16) attend_few<ST, D, 1>(a, pl, w, even, odd);
            else attend_few<ST, D, 2>(a, pl, w, even, odd);
            w = then;
        }
    }
}

// ---- the join --------------------------------------------------------------------------------------------------
// Records are joined by groups of D / 4 threads, 16 bytes of the row a thread.
template <typename ST, int D>
struct Join {
    static constexpr int C4 = D / 4;
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
    // every step-th record of row r of a tile, from the lo-th on; whole: the row's own record
    template <bool MANY>
    __device__ __forceinline__ void add_tile(const PagedParams &a, const Span &s, int r, long whole, int lo, int step, int c4)
    {
        constexpr int AHEAD = 4;  // records on their way together
        const bool one = s.w0 == s.w1;
        for (int w = s.w0 + lo; w <= s.w1; w += AHEAD * step) {
            float2 ml[AHEAD];
            f32x4 v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int x = w + i * step;
                ml[i] = make_float2(-INFINITY, 0.f);
                v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (x <= s.w1) {
                    const long at = one ? whole : cut_row(a, MANY, x, x == s.w0 ? s.begun : 0) + r;
                    ml[i] = *reinterpret_cast<const float2 *>((one ? a.row_ml : a.cut_ml) + at * 2);
                    v[i] = *reinterpret_cast<const f32x4 *>((one ? a.row_o : a.cut_o) + at * D + 4 * c4);
                }
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) add(ml[i].x, ml[i].y, v[i]);
        }
    }
    __device__ __forceinline__ void put(const PagedParams &a, long row, int c4) const
    {
        TileWork w;
        w.direct = true;
        put4<ST, D>(a, w, row, 0, 4 * c4, o, m, l);
    }
};

// Where a sequence's rows are one tile: a wave for every row, the records divided among its 2 or 4 groups.  Nothing but trips to memory
// (the entry, the records), so many waves and little arithmetic: with the spans worked out here by every wave the join of 2048 rows took 16 us
// instead of 7.
template <typename ST, int D>
__global__ __launch_bounds__(64) void paged_join_rows_kernel(const PagedParams a)
{
    using J = Join<ST, D>;
    constexpr int NG = 64 / J::C4;
    const int c4 = threadIdx.x % J::C4, grp = threadIdx.x / J::C4;
    const int rows = a.B * a.Hq * a.T;
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const int bh = row / a.T, t = row - bh * a.T, b = bh / a.Hq, hq = bh - b * a.Hq, kvh = hq / a.G, r = t * a.G + hq - kvh * a.G;
        const JoinEntry e = a.entries[b * a.Hkv + kvh];
        if (t >= e.n) continue;
        const bool none = e.shared[0].w1 < e.shared[0].w0;
        if (none && e.own.w0 == e.own.w1) continue;  // written as it is
        J j;
        if (a.own_many) j.template add_tile<true>(a, e.own, r, (long)rows + row, NG - 1 - grp, NG, c4);
        else j.template add_tile<false>(a, e.own, r, (long)rows + row, NG - 1 - grp, NG, c4);
        if (!none) {
            const int in = e.row0 + r;
            if (e.many) j.template add_tile<true>(a, e.shared[in >= kMany], in % kMany, row, grp, NG, c4);
            else j.template add_tile<false>(a, e.shared[in >= kFew], in % kFew, row, grp, NG, c4);
        }
        J sum;  // in the order of the groups, the same in all of them
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            f32x4 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = shfl_f(j.o[k], i * J::C4 + c4);
            sum.add(shfl_f(j.m, i * J::C4), shfl_f(j.l, i * J::C4), o);
        }
        if (grp == 0) sum.put(a, row, c4);
    }
}

// Where they are many: only the tiles that the line's cuts go through, workgroups i looking at the end of the i-th share; and the rows that see
// nothing, which may have no tile.
template <typename ST, int D, bool MANY>
__global__ __launch_bounds__(kPagedThreads) void paged_join_cuts_kernel(const PagedParams a)
{
    using J = Join<ST, D>;
    constexpr int ROWS = MANY ? kMany : kFew, NG = kPagedThreads / J::C4;
    const Plan pl(a.plan + kPlanShares, a.B);
    const int c4 = threadIdx.x % J::C4, grp = threadIdx.x / J::C4;
    for (int b = blockIdx.x; blockIdx.y == 0 && b < a.B; b += gridDim.x) {
        const int none = min(pl.seq[b].n - pl.seq[b].L, pl.seq[b].n);
        for (int e = grp; e < none * a.Hq; e += NG) {
            J j;
            j.put(a, (long)(b * a.Hq + e / none) * a.T + e % none, c4);
        }
    }
    const Shares sh = *reinterpret_cast<const Shares *>(a.plan + (MANY ? kPlanShares / 2 : 0));
    if ((int)blockIdx.x + 1 >= sh.n) return;
    const long cut = sh.begin(blockIdx.x + 1);
    TileWork w;
    long s0, s1;
    find_tile<ST>(a, pl, kind_of<ST>(MANY), cut, sh.line, w, s0, s1);
    if (cut <= s0 || sh.begin(blockIdx.x) > s0) return;  // not through its units; not its first
    const int rows = min(w.rows - w.rt * ROWS, ROWS);
    const Span span = span_of(sh, s0, (int)(s1 - s0));
    for (int r = blockIdx.y * NG + grp; r < rows; r += gridDim.y * NG) {
        int bq, t, g;
        if (!query_of(a, pl, w, w.rt * ROWS + r, bq, t, g)) continue;
        J j;
        j.template add_tile<MANY>(a, span, r, 0, 0, 1, c4);
        j.put(a, out_row(a, w, bq, t, g), c4);
    }
}

int check_pool(const rs_pool *p);  // pool.hip

static int tile_rows(const rs_shape *s) { return s->dtype == RS_BF16 ? kMany : kFew; }

struct PagedLayout {
    bool own_many, shares;   // a sequence's own tiles are of many rows; rows of several sequences may be put together
    int few_rows;            // rows of a few-row tile, at most
    int groups;              // of the first launch
    size_t many, cut, rows;  // boundary records' rows of many-row tiles, of both kinds; row records
    size_t off_ml, off_plan, total;
};
static PagedLayout paged_layout(const rs_shape *s, int T_new)
{
    PagedLayout x;
    const long own = (long)T_new * (s->Hq / s->Hkv);
    // Rows of several sequences are put together only where one sequence's rows leave room in a tile; else a
    // tile's rows come from one sequence anyway and its keys are one segment, without records to join.
    x.shares = own < tile_rows(s);
    const long most = x.shares ? own * s->B : own;
    x.own_many = s->dtype == RS_BF16 && own > kFew;
    x.few_rows = (int)(most < kFew ? most : kFew);
    // (three of 49.4 KB and 36 bytes an entry in the 160 KB of a CU; of longer lists, two)
    x.groups = x.own_many && s->B <= 112 ? kManyGroups : kPagedGroups;
    x.many = (s->dtype == RS_BF16 && most > kFew) ? (size_t)2 * x.groups * kMany : 0;
    x.cut = x.many + (x.own_many ? 0 : (size_t)2 * kPagedGroups * kPagedWaves * x.few_rows);
    x.rows = x.shares ? (size_t)s->B * s->Hq * T_new * 2 : 0;
    x.off_ml = RS_WS_CTRL_BYTES + align256((x.cut + x.rows) * s->D * 4);
    x.off_plan = x.off_ml + align256((x.cut + x.rows) * 8);
    x.total = x.off_plan + kPlanShares + plan_room(s->B) + align256((size_t)s->B * s->Hkv * sizeof(JoinEntry));
    return x;
}

static int check_paged(const rs_shape *s, const rs_pool *p, int T_new)
{
    int st = check_rows(s, true);
    if (st == RS_OK) st = check_pool(p);
    if (st != RS_OK) return st;
    if (p->P != s->P || (long)p->N * p->P != s->Tcap || T_new < 1) return RS_INVALID_ARG;
    if (s->B > kMaxList) return RS_UNSUPPORTED;
    // places of a KV head's line, at most: they are counted in 32 bits
    const double own = (double)T_new * (s->Hq / s->Hkv), tokens = (double)p->M * p->P;
    const double few = s->B * (own / kFew + 2) * (tokens / (s->dtype == RS_BF16 ? kKeys<bf16> : kKeys<float>) + 3);
    const double many = s->B * (own / kMany + 2) * (tokens / 128 + 2);
    if ((paged_layout(s, T_new).own_many ? many : few) * 2 > 2e9 || (double)s->B * s->Hq * T_new > 2e9) return RS_UNSUPPORTED;
    return RS_OK;
}

template <typename ST, int D>
static void paged_launch(const PagedParams &a, hipStream_t stream)
{
    if (sizeof(ST) == 2 && a.own_many) paged_attend_kernel<ST, D, sizeof(ST) == 2><<<a.groups, kPagedThreads, plan_bytes(a.B), stream>>>(a);
    else paged_attend_kernel<ST, D, false><<<a.groups, kPagedThreads, plan_bytes(a.B), stream>>>(a);
    const long rows = (long)a.B * a.Hq * a.T;
    // (workgroups a cut few-row tile 1 / 2 / 4, float32, 16 heads over 8, us: 24 tokens each of 4 after 600 to 900 51.9 / 45.4 / 43.7, of 8 59.2 / 53.3 / 53.7,
    // 100 each of 8 after 2000 to 3000 195 / 195 / 204)
    if (a.entries) paged_join_rows_kernel<ST, D><<<(unsigned)(rows < 8192 ? rows : 8192), 64, 0, stream>>>(a);
    else if (sizeof(ST) == 2) paged_join_cuts_kernel<ST, D, true><<<dim3((unsigned)a.groups, 4), kPagedThreads, 0, stream>>>(a);
    else paged_join_cuts_kernel<ST, D, false><<<dim3(kPagedGroups * kPagedWaves, 2), kPagedThreads, 0, stream>>>(a);
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
    a.share = x.shares ? share : nullptr;
    a.out = out, a.lse = lse_out;
    a.cut_o = (float *)((char *)ws + RS_WS_CTRL_BYTES), a.row_o = a.cut_o + x.cut * s->D;
    a.cut_ml = (float *)((char *)ws + x.off_ml), a.row_ml = a.cut_ml + x.cut * 2;
    a.plan = (char *)ws + x.off_plan;
    a.entries = x.shares ? (JoinEntry *)(a.plan + kPlanShares + plan_room(s->B)) : nullptr;
    a.few_base = (long)x.many, a.few_rows = x.few_rows, a.own_many = x.own_many, a.groups = x.groups;
    a.B = s->B, a.Hq = s->Hq, a.Hkv = s->Hkv, a.G = s->Hq / s->Hkv;
    a.S = p->S, a.M = p->M, a.N = p->N, a.shift = __builtin_ctz((unsigned)p->P), a.T = T_new;
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
