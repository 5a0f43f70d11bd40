// Dense attention of the newest tokens of many sequences over a pool of pages, the pages that neighbours of the list have in
// common read once for all of them (Eq. 4 with every token).
//
// Mathematics.  With z_j = scale q . k_j and any split of the positions into parts, each part leaves m = max z_j, l = sum e^(z_j - m),
// o = sum e^(z_j - m) v_j, and parts join by m = max m_i, (l, o) = sum e^(m_i - m) (l_i, o_i): the shared pages are one
// part, attended by the rows of all sequences of the run at once, a sequence's own pages another, and each is split
// further along its keys for balance.
//
// Work.  Segments (a run's shared pages, a sequence's own pages) times tiles of up to kRows query rows, each cut into units of 4 KT keys;
// per KV head the units of all segments form one line, the lines of the heads another, and every workgroup takes an equal
// share of it, whatever the lengths are.  Where that line is cut and which unit belongs to whom follows from the lengths alone: each workgroup
// works it out for itself (a prefix sum over the list), so lengths live on the device and nothing has to be planned by the host.
// What a workgroup holds of a tile goes to one of its two boundary records if the tile goes on elsewhere, to the row's record
// if it has a second part (shared and own), else straight to the output; a second launch joins the records.
//
// A workgroup's four waves take KT keys each of a unit (own LDS, own softmax state, no barrier in the loop) and join at the end of a
// tile.  S^T = K Q^T and O^T = V^T P^T by 16-wide matrix instructions: a lane holds the keys of one query, P^T goes
// from the accumulators into the second product as it is.  K and V arrive by direct global -> LDS loads, the next K tile while the softmax and the
// second product run, the next V tile while the next scores are formed.
#include "check.h"
#include "common.h"

namespace rs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
constexpr int kMaxList = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // the softmax's reference point moves when the maximum has grown by more (base-2 exponent)

// keys a wave takes at a time, and 16-row tiles of queries it can hold (registers: float32 queries take twice as many)
template <typename ST>
struct PagedTile;
template <>
struct PagedTile<bf16> {
    static constexpr int KT = 32, MAXRT = 2;
};
template <>
struct PagedTile<float> {
    static constexpr int KT = 16, MAXRT = 2;
};

struct PagedParams {
    const void *q, *k, *v;
    const int32_t *table, *len, *seq, *n_new, *share;
    void *out;
    float *lse;
    float *cut_o, *cut_ml;      // boundary records: [2 workgroups][rows of a tile] x D, x 2
    float *row_o, *row_ml;      // row records: [shared, own][B Hq T] x D, x 2; nullptr: no segment is shared
    int B, Hq, Hkv, G, S, M, N, shift, T, groups;
    float scale;
};

// The line of units of one KV head, in LDS: `seqs` int4 and 3 B + 1 words.
struct Seq {
    int L, n, c, first;  // tokens, new ones, pages of the run's shared part (0: none), the run's first place
};
struct Plan {
    Seq *seq;      // [B]
    int *start;    // [B + 1] units before this place of the list
    int *members;  // [B] members of the run that begins here (0: none begins, or it shares nothing)
    int *fewest;   // [B] pages a run can share
    __device__ __forceinline__ Plan(char *lds, int B) : seq((Seq *)lds), start((int *)(seq + B)), members(start + B + 1), fewest(members + B) {}
};
static size_t plan_bytes(int B) { return (size_t)B * 16 + (size_t)(3 * B + 1) * 4; }

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }

// units of row tile rt of sequence x over its own pages: the keys from the shared ones to the tile's last row
template <int ROWS, int UNIT>
__device__ __forceinline__ int own_units(const Seq &x, int rt, int G, int shift, int &k0, int &k1)
{
    const int t0 = rt * ROWS / G, t1 = min(x.n - 1, (rt * ROWS + ROWS - 1) / G);
    k0 = x.c << shift;
    k1 = x.L - x.n + t1 + 1;
    return (t0 >= x.n || k1 <= k0) ? 0 : (k1 - k0 + UNIT - 1) / UNIT;
}
template <int ROWS>
__device__ __forceinline__ int shared_tiles(int members, int T, int G) { return div_up(members * T * G, ROWS); }

// Fills the plan; called by the whole workgroup (kPagedThreads).
template <int ROWS, int UNIT>
__device__ __forceinline__ void make_plan(const PagedParams &a, const Plan &pl)
{
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
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += kPagedThreads) atomicMin(&pl.fewest[pl.seq[b].first], pl.seq[b].c);
    __syncthreads();
    // (a thread's stretch of the list, so that a second pass can add what precedes it)
    const int each = div_up(a.B, kPagedThreads), lo = min(tid * each, a.B), hi = min(lo + each, a.B);
    int sum = 0;
    for (int b = lo; b < hi; ++b) {
        const int f = pl.seq[b].first;
        const int c = pl.members[f] ? pl.fewest[f] : 0;  // (nobody writes members or first here)
        int units = 0, k0, k1;
        const Seq x{pl.seq[b].L, pl.seq[b].n, c, f};
        if (f == b && c > 0) units += shared_tiles<ROWS>(pl.members[b], a.T, a.G) * div_up(c << a.shift, UNIT);
        for (int rt = 0; rt * ROWS < x.n * a.G; ++rt) units += own_units<ROWS, UNIT>(x, rt, a.G, a.shift, k0, k1);
        pl.start[b] = units;
        sum += units;
    }
    __syncthreads();
    for (int b = lo; b < hi; ++b) {
        const int f = pl.seq[b].first;
        pl.seq[b].c = pl.members[f] ? pl.fewest[f] : 0;
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

// where a tile's part in workgroup w goes: 2: all of the tile is here; 0, 1: a boundary record
__device__ __forceinline__ int record_of(long s0, long s1, long wb, long we) { return (s0 >= wb && s1 <= we) ? 2 : s0 <= wb ? 0 : 1; }

// ---- operands ---------------------------------------------------------------------------------------------------
// Rows lie unpadded in LDS, the 16-byte chunks of each permuted so that operand reads touch every bank once: for K, 16 lanes
// read the same chunk of 16 rows; for V (bfloat16) 32 lanes read two chunks of each of 8 rows, (float32) 64 lanes four
// chunks of each of 4 rows, 4 apart.
template <typename ST, int D>
struct PagedRows {
    static constexpr int ROW = D * (int)sizeof(ST), CR = ROW / 16, RW = 64 / CR, NL = 16 / RW;  // chunks a row, rows and loads a wave
    __device__ __forceinline__ static int k_swizzle(int row) { return CR >= 16 ? row & 15 : (row >> 1) & 7; }
    __device__ __forceinline__ static int v_swizzle(int row)
    {
        if (sizeof(ST) == 4) return 4 * ((row >> 2) & 3);
        return CR == 16 ? 2 * (row & 7) : 2 * ((row >> 1) & 3);
    }
    // 16 rows from a descriptor that ends with the last valid one into LDS
    template <bool V>
    __device__ __forceinline__ static void load(LdsSource src, char *tile)
    {
        const int lane = lane_id();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = i * RW + lane / CR, chunk = (lane % CR) ^ (V ? v_swizzle(row) : k_swizzle(row));
            load16_to_lds_at(src, (uint32_t)(row * ROW + chunk * 16), 0u, tile + i * 1024);
        }
    }
};

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

// one tile of rows over a run of keys
struct TileWork {
    int kvh, b, rt, rows;     // rows: of the segment (the tile takes those from rt * ROWS on)
    bool shared;
    int row_seq;              // whose table row names the pages
    int key0, units, limit;   // first key, units of keys from there, keys that exist (later ones are nobody's)
    int record;               // record_of()
    long slot;                // of the boundary record
    bool direct;              // a whole tile without a second part
};

// the query behind row r of a segment: false: none
__device__ __forceinline__ bool query_of(const PagedParams &a, const Plan &pl, bool shared, int b, int r, int rows, int &bq, int &t, int &g)
{
    if (r >= rows) return false;
    const int per = a.T * a.G;
    bq = b;
    if (shared) {
        bq = b + r / per;
        r %= per;
    }
    t = r / a.G;
    g = r % a.G;
    return t < pl.seq[bq].n;
}

template <typename ST, int D, int RT>
__device__ __forceinline__ void attend_tile(const PagedParams &a, const Plan &pl, const TileWork &w, char *sK, char *sV, float *s_m, float *s_l)
{
    using Rows = PagedRows<ST, D>;
    constexpr bool BF = sizeof(ST) == 2;
    constexpr int KT = PagedTile<ST>::KT, NH = KT / 16, ROWS = 16 * PagedTile<ST>::MAXRT;
    constexpr int NDT = D / 16, NL = Rows::NL * NH;       // 16-channel tiles of O^T; loads of a step's K (or V)
    constexpr int NK = BF ? D / 32 : D / 16;              // operand registers groups of a query
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;
    char *cK = sK + wave * (KT * Rows::ROW), *cV = sV + wave * (KT * Rows::ROW);

    // ---- pages of this wave's steps ----
    const int32_t *trow = a.table + (long)w.row_seq * a.M;
    const ST *kb = (const ST *)a.k + (long)w.kvh * ((long)a.N << a.shift) * D, *vb = (const ST *)a.v + (long)w.kvh * ((long)a.N << a.shift) * D;
    const int base = w.key0 + wave * KT, in_page = (1 << a.shift) - 1;
    auto key_of = [&](int n) { return base + (n / NH) * (kPagedWaves * KT) + (n % NH) * 16; };  // of the wave's n-th 16 keys
    auto fetch = [&](int n) {
        const int key = key_of(n);
        int page = -1;
        if (n < w.units * NH && key < w.limit) page = trow[key >> a.shift];
        return (page < 0 || page >= a.N) ? -1 : page;
    };
    int listed = -1, taken = 0;
    struct Step {
        LdsSource k[NH], v[NH];
        int valid[NH];
    };
    auto next_step = [&](Step &x) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            if ((taken & 63) == 0) {
                listed = fetch(taken + lane);
                asm volatile("" : "+v"(listed));  // (waited for here, and not by every step)
            }
            const int page = __builtin_amdgcn_readlane(listed, taken & 63), key = key_of(taken);
            const int left = w.limit - key;
            x.valid[h] = page < 0 ? 0 : left < 16 ? max(left, 0) : 16;
            const long at = page < 0 ? 0 : ((((long)page << a.shift) + (key & in_page)) * D);
            x.k[h] = lds_source_sized(kb + at, x.valid[h] * Rows::ROW);
            x.v[h] = lds_source_sized(vb + at, x.valid[h] * Rows::ROW);
            ++taken;
        }
    };
    Step cur;
    next_step(cur);
#pragma unroll
    for (int h = 0; h < NH; ++h) Rows::template load<false>(cur.k[h], cK + h * 16 * Rows::ROW);
#pragma unroll
    for (int h = 0; h < NH; ++h) Rows::template load<true>(cur.v[h], cV + h * 16 * Rows::ROW);

    // ---- this lane's queries ----
    f32x4 qf[RT][NK];  // bfloat16: 8 channels a register group, float32: 4
    int last[RT];      // the last position the row sees (-1: there is no such row)
    int first_last = 0x7fffffff;  // the smallest of the tile's rows
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        int bq, t, g;
        const bool real = query_of(a, pl, w.shared, w.b, w.rt * ROWS + rt * 16 + l16, w.rows, bq, t, g);
        last[rt] = -1;
        const ST *q = (const ST *)a.q;
        if (real) {
            q += ((long)(bq * a.Hq + w.kvh * a.G + g) * a.T + t) * D;
            last[rt] = pl.seq[bq].L - pl.seq[bq].n + t;
        }
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(q + (BF ? 32 * kk + 8 * lg : 16 * kk + 4 * lg));
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
    const int k_sw = Rows::k_swizzle(l16);

    for (int u = 0; u < w.units; ++u) {
        const int key = base + u * (kPagedWaves * KT);
        const bool more = u + 1 < w.units;
        // ---- S^T = K Q^T: lane (l16, lg) gets keys 4 lg .. 4 lg + 3 of every 16 for query l16 ----
        wait_loads<NL>();  // K is here (V, issued after it, may be on its way)
        f32x4 s[RT][NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                const f32x4 kf = *reinterpret_cast<const f32x4 *>(cK + (16 * h + l16) * Rows::ROW + (((4 * kk + lg) ^ k_sw) * 16));
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if constexpr (BF) {
                        s[rt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[rt][kk]),
                                                                          s[rt][h], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[rt][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j], qf[rt][kk][j], s[rt][h], 0, 0, 0);
                    }
                }
            }
        }
        wait_lds_reads();
        const bool whole = cur.valid[0] == 16 && cur.valid[NH - 1] == 16;
        int valid[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) valid[h] = cur.valid[h];
        if (more) {
            next_step(cur);
#pragma unroll
            for (int h = 0; h < NH; ++h) Rows::template load<false>(cur.k[h], cK + h * 16 * Rows::ROW);
        }
        // ---- softmax, base 2 ----
        const bool edge = key + KT - 1 > first_last;  // some row does not see some key of this step
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = -INFINITY;
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float z = s[rt][h][i] * cs;
                    if (!whole || edge) {
                        const int n = 4 * lg + i;
                        if (n >= valid[h] || (edge && key + 16 * h + n > last[rt])) z = -INFINITY;
                    }
                    s[rt][h][i] = z;
                    mx = fmaxf(mx, z);
                }
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
        if (more) wait_loads<NL>();
        else wait_loads<0>();
        bool odd = false;  // a value that is not finite where some row may not look
        if constexpr (BF) {
            bf16x8 pf[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 8; ++i) pf[rt][i] = (__bf16)s[rt][i / 4][i % 4];
            union Vf {
                s16x4 h[2];
                bf16x8 f;
            };
            auto v_of = [&](int dt) __attribute__((always_inline)) {
                Vf vf;
                const int row = 4 * lg + (l16 >> 2), chunk = 2 * dt + ((l16 & 3) >> 1);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    vf.h[h] = paged_read_tr16(cV + (16 * h + row) * Rows::ROW + ((chunk ^ Rows::v_swizzle(row)) * 16) + 8 * (l16 & 1));
                return vf;
            };
            if (edge) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    const Vf vf = v_of(dt);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i) odd |= (vf.h[h][i] & 0x7f80) == 0x7f80;
                }
                odd = __any(odd);
            }
            if (!odd) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    const Vf vf = v_of(dt);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) oacc[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.f, pf[rt], oacc[rt][dt], 0, 0, 0);
                }
            }
        } else {
            // lane (l16, lg) reads channel 16 dt + l16 of rows 4 lg + j
            auto v_of = [&](int dt, int j) __attribute__((always_inline)) {
                const int row = 4 * lg + j, chunk = 4 * dt + (l16 >> 2);
                return *reinterpret_cast<const float *>(cV + row * Rows::ROW + ((chunk ^ Rows::v_swizzle(row)) * 16) + 4 * (l16 & 3));
            };
            if (edge) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= (__float_as_uint(v_of(dt, j)) & 0x7f800000u) == 0x7f800000u;
                odd = __any(odd);
            }
            if (!odd) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float vf = v_of(dt, j);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) oacc[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, s[rt][0][j], oacc[rt][dt], 0, 0, 0);
                    }
            }
        }
        if (odd) {
            // An infinity or NaN among values that some row is not to see (0 times it would be NaN): key by key, only into
            // the rows that see it.
#pragma unroll 1
            for (int n = 0; n < KT; ++n) {
                const char *vrow = cV + n * Rows::ROW;
                const int sw = Rows::v_swizzle(n & 15);
                float p[RT];
                bool sees[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    p[rt] = 0.f;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = shfl_f(s[rt][h][i], ((n & 15) >> 2) * 16 + l16);
                            if (h == n >> 4 && i == (n & 3)) p[rt] = x;
                        }
                    sees[rt] = key + n <= last[rt];  // (rows that do not exist, and keys of missing pages: zeros)
                }
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = (16 * dt + 4 * lg + i) * (int)sizeof(ST);
                        const float y = to_f32(*reinterpret_cast<const ST *>(vrow + (((at >> 4) ^ sw) << 4) + (at & 15)));
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            if (sees[rt]) oacc[rt][dt][i] = fmaf(p[rt], y, oacc[rt][dt][i]);
                    }
            }
        }
        wait_lds_reads();
        if (more) {
#pragma unroll
            for (int h = 0; h < NH; ++h) Rows::template load<true>(cur.v[h], cV + h * 16 * Rows::ROW);
        }
    }

    // ---- the four waves' parts become one ----
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float sum = quad_sum(l[rt]);
        if (lg == 0) {
            s_m[wave * ROWS + rt * 16 + l16] = m[rt];
            s_l[wave * ROWS + rt * 16 + l16] = sum;
        }
    }
    constexpr int C4 = D / 4;  // 16-byte columns of an output row
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        f32x4 *mine = reinterpret_cast<f32x4 *>(cK);  // 16 rows of D floats: a step's K rows are as large
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) mine[l16 * C4 + ((4 * dt + lg) ^ l16)] = oacc[rt][dt];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * C4; e += kPagedThreads) {
            const int r = e / C4, c4 = e % C4;
            int bq, t, g;
            if (!query_of(a, pl, w.shared, w.b, w.rt * ROWS + rt * 16 + r, w.rows, bq, t, g)) continue;
            float mw[kPagedWaves], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kPagedWaves; ++i) {
                mw[i] = s_m[i * ROWS + rt * 16 + r];
                top = fmaxf(top, mw[i]);
            }
            float L = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kPagedWaves; ++i) {
                if (mw[i] == -INFINITY && s_l[i * ROWS + rt * 16 + r] == 0.f) continue;  // saw nothing
                const float f = mw[i] == top ? 1.f : __builtin_amdgcn_exp2f(mw[i] - top);
                L = fmaf(f, s_l[i * ROWS + rt * 16 + r], L);
                const f32x4 x = *(reinterpret_cast<const f32x4 *>(sK + i * (KT * Rows::ROW)) + r * C4 + (c4 ^ r));
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(f, x[j], o[j]);
            }
            const long row = (long)(bq * a.Hq + w.kvh * a.G + g) * a.T + t;
            if (w.direct) {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                ST y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) from_f32(y[j], o[j] * inv);
                __builtin_memcpy((ST *)a.out + row * D + 4 * c4, y, sizeof(y));
                if (a.lse && c4 == 0) a.lse[row] = L == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(L)) * kLn2;
            } else {
                const long at = w.record == 2 ? (w.shared ? 0 : (long)a.B * a.Hq * a.T) + row : w.slot * ROWS + rt * 16 + r;
                float *po = (w.record == 2 ? a.row_o : a.cut_o) + at * D, *ml = (w.record == 2 ? a.row_ml : a.cut_ml) + at * 2;
                *reinterpret_cast<f32x4 *>(po + 4 * c4) = o;
                if (c4 == 0) {
                    ml[0] = top;
                    ml[1] = L;
                }
            }
        }
        __syncthreads();
    }
}

template <typename ST, int D>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_attend_kernel(const PagedParams a)
{
    constexpr int KT = PagedTile<ST>::KT, ROWS = 16 * PagedTile<ST>::MAXRT, UNIT = kPagedWaves * KT;
    __shared__ __attribute__((aligned(1024))) char sK[kPagedWaves * KT * D * sizeof(ST)];
    __shared__ __attribute__((aligned(1024))) char sV[kPagedWaves * KT * D * sizeof(ST)];
    __shared__ float s_m[kPagedWaves * ROWS], s_l[kPagedWaves * ROWS];
    extern __shared__ __attribute__((aligned(16))) char lds_plan[];
    const Plan pl(lds_plan, a.B);
    make_plan<ROWS, UNIT>(a, pl);
    const int line = pl.start[a.B];
    const long all = (long)line * a.Hkv, each = (all + gridDim.x - 1) / gridDim.x;
    const long wb = each * blockIdx.x, we = min(wb + each, all);
    for (long at = wb; at < we;) {
        TileWork w;
        w.kvh = (int)(at / line);
        int off = (int)(at % line);
        int lo = 0, hi = a.B;  // the last place whose units begin at or before off (places without units are passed over)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (pl.start[mid] <= off) lo = mid;
            else hi = mid;
        }
        w.b = lo;
        off -= pl.start[lo];
        const Seq x = pl.seq[lo];
        const int su = (x.first == lo && x.c > 0) ? div_up(x.c << a.shift, UNIT) : 0;
        const int st = su ? shared_tiles<ROWS>(pl.members[lo], a.T, a.G) : 0;
        int n, k0, k1;
        w.shared = off < su * st;
        if (w.shared) {
            w.rt = off / su;
            off -= w.rt * su;
            n = su;
            k0 = 0;
            k1 = x.c << a.shift;
            w.rows = pl.members[lo] * a.T * a.G;
        } else {
            off -= su * st;
            w.rt = 0;
            w.rows = x.n * a.G;
            while (off >= (n = own_units<ROWS, UNIT>(x, w.rt, a.G, a.shift, k0, k1))) {
                off -= n;
                ++w.rt;
            }
        }
        const long s0 = at - off, s1 = s0 + n;
        w.row_seq = a.seq[lo];
        w.key0 = k0 + off * UNIT;
        w.units = (int)min((long)(n - off), we - at);
        w.limit = k1;
        w.record = record_of(s0, s1, wb, we);
        w.slot = 2l * blockIdx.x + (w.record & 1);
        w.direct = w.record == 2 && !w.shared && x.c == 0;
        const int rows = min(ROWS, w.rows - w.rt * ROWS);
        if (rows <= 16) attend_tile<ST, D, 1>(a, pl, w, sK, sV, s_m, s_l);
        else if (rows <= 32 || PagedTile<ST>::MAXRT == 2) attend_tile<ST, D, 2>(a, pl, w, sK, sV, s_m, s_l);
        else attend_tile<ST, D, PagedTile<ST>::MAXRT>(a, pl, w, sK, sV, s_m, s_l);
        at += w.units;
    }
}

// Joins the records of every row that was not written at once: a workgroup for each row, 16 bytes of the row a thread, the records
// divided among the 4 x 64 / (D / 4) thread groups.
template <typename ST, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_join_kernel(const PagedParams a)
{
    constexpr int KT = PagedTile<ST>::KT, ROWS = 16 * PagedTile<ST>::MAXRT, UNIT = kPagedWaves * KT;
    constexpr int C4 = D / 4, NG = kPagedThreads / C4;
    __shared__ float s_m[NG], s_l[NG];
    __shared__ f32x4 s_o[NG][C4];
    extern __shared__ __attribute__((aligned(16))) char lds_plan[];
    const Plan pl(lds_plan, a.B);
    make_plan<ROWS, UNIT>(a, pl);
    const int line = pl.start[a.B], c4 = threadIdx.x % C4, grp = threadIdx.x / C4;
    const long all = (long)line * a.Hkv, each = max((all + a.groups - 1) / a.groups, 1l);
    const long rows = (long)a.B * a.Hq * a.T;
    for (long row = blockIdx.x; row < rows; row += gridDim.x) {
        const int t = (int)(row % a.T), hq = (int)(row / a.T % a.Hq), b = (int)(row / a.T / a.Hq);
        const Seq x = pl.seq[b];
        if (t >= x.n) continue;
        const int kvh = hq / a.G, g = hq % a.G;
        float m = -INFINITY, l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        bool written = false;
        for (int part = 0; part < 2; ++part) {  // own, shared
            const bool shared = part == 1;
            if (shared && x.c == 0) break;
            const int lead = shared ? x.first : b, r = shared ? ((b - lead) * a.T + t) * a.G + g : t * a.G + g, rt = r / ROWS;
            const Seq y = pl.seq[lead];
            const int su = (y.first == lead && y.c > 0) ? div_up(y.c << a.shift, UNIT) : 0;
            int k0, k1, n = su;
            long s0 = (long)kvh * line + pl.start[lead];
            if (shared) {
                s0 += (long)rt * su;
            } else {
                s0 += su ? (long)su * shared_tiles<ROWS>(pl.members[lead], a.T, a.G) : 0l;
                for (int i = 0; i < rt; ++i) s0 += own_units<ROWS, UNIT>(y, i, a.G, a.shift, k0, k1);
                n = own_units<ROWS, UNIT>(y, rt, a.G, a.shift, k0, k1);
            }
            if (n == 0) continue;
            const long w0 = s0 / each, w1 = (s0 + n - 1) / each;
            if (w0 == w1 && !shared && x.c == 0) {
                written = true;
                break;
            }
            for (long w = w0 + grp; w <= w1; w += NG) {
                const int rec = record_of(s0, s0 + n, w * each, min(w * each + each, all));
                const long at = rec == 2 ? (shared ? 0 : rows) + row : (2 * w + rec) * ROWS + r % ROWS;
                const float *ml = (rec == 2 ? a.row_ml : a.cut_ml) + at * 2;
                const f32x4 v = *reinterpret_cast<const f32x4 *>((rec == 2 ? a.row_o : a.cut_o) + at * D + 4 * c4);
                const float m1 = ml[0], l1 = ml[1];
                if (m1 == -INFINITY && l1 == 0.f) continue;
                const float top = fmaxf(m, m1), f0 = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), f1 = m1 == top ? 1.f : __builtin_amdgcn_exp2f(m1 - top);
                m = top;
                l = l * f0 + l1 * f1;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = o[j] * f0 + v[j] * f1;
            }
        }
        if (written) continue;  // (the same for the whole workgroup)
        if (c4 == 0) {
            s_m[grp] = m;
            s_l[grp] = l;
        }
        s_o[grp][c4] = o;
        __syncthreads();
        if (grp == 0) {
            float top = -INFINITY, L = 0.f;
#pragma unroll
            for (int i = 0; i < NG; ++i) top = fmaxf(top, s_m[i]);
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                if (s_m[i] == -INFINITY && s_l[i] == 0.f) continue;
                const float f = s_m[i] == top ? 1.f : __builtin_amdgcn_exp2f(s_m[i] - top);
                L = fmaf(f, s_l[i], L);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = fmaf(f, s_o[i][c4][j], y[j]);
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            ST z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) from_f32(z[j], y[j] * inv);
            __builtin_memcpy((ST *)a.out + row * D + 4 * c4, z, sizeof(z));
            if (a.lse && c4 == 0) a.lse[row] = L == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(L)) * kLn2;
        }
        __syncthreads();
    }
}

int check_pool(const rs_pool *p);  // pool.hip

constexpr int kPagedGroups = 512;  // two workgroups a CU

static int tile_rows(int dtype) { return 16 * (dtype == RS_BF16 ? PagedTile<bf16>::MAXRT : PagedTile<float>::MAXRT); }
static int unit_keys(int dtype) { return kPagedWaves * (dtype == RS_BF16 ? PagedTile<bf16>::KT : PagedTile<float>::KT); }

// Whether the rows of several sequences are put together: only where one sequence's rows leave room in a tile; else a
// tile's rows come from one sequence anyway and its keys are one segment, without records to join.
static bool rows_are_shared(const rs_shape *s, int T_new) { return (long)T_new * (s->Hq / s->Hkv) < tile_rows(s->dtype); }

static size_t paged_ws(const rs_shape *s, int T_new, size_t *cut_rows, size_t *rows)
{
    *cut_rows = (size_t)2 * kPagedGroups * tile_rows(s->dtype);
    *rows = rows_are_shared(s, T_new) ? (size_t)s->B * s->Hq * T_new * 2 : 0;
    return RS_WS_CTRL_BYTES + align256((*cut_rows + *rows) * s->D * 4) + align256((*cut_rows + *rows) * 8);
}

static int check_paged(const rs_shape *s, const rs_pool *p, int T_new)
{
    int st = check_shape(s, true);
    if (st == RS_OK) st = check_pool(p);
    if (st != RS_OK) return st;
    if (p->P != s->P || (long)p->N * p->P != s->Tcap || T_new < 1) return RS_INVALID_ARG;
    if (s->B > kMaxList) return RS_UNSUPPORTED;
    // units of a KV head's line, at most: they are counted in 32 bits
    const double tiles = (double)s->B * ((double)T_new * (s->Hq / s->Hkv) / tile_rows(s->dtype) + 2);
    if (tiles * ((double)p->M * p->P / unit_keys(s->dtype) + 1) * 2 > 2e9 || (double)s->B * s->Hq * T_new > 2e9) return RS_UNSUPPORTED;
    return RS_OK;
}

template <typename ST, int D>
static void paged_launch(const PagedParams &a, hipStream_t stream)
{
    const size_t lds = plan_bytes(a.B);
    paged_attend_kernel<ST, D><<<(unsigned)a.groups, kPagedThreads, lds, stream>>>(a);
    const long rows = (long)a.B * a.Hq * a.T;
    paged_join_kernel<ST, D><<<(unsigned)(rows < 2048 ? rows : 2048), kPagedThreads, lds, stream>>>(a);
}

}  // namespace rs

using namespace rs;

extern "C" {

size_t attn_paged_workspace_bytes(const rs_shape *s, const rs_pool *p, int32_t T_new)
{
    size_t cut, rows;
    return check_paged(s, p, T_new) == RS_OK ? paged_ws(s, T_new, &cut, &rows) : 0;
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
    size_t cut, rows;
    if (!ws || !aligned16(ws) || ws_bytes < paged_ws(s, T_new, &cut, &rows)) return RS_WORKSPACE_TOO_SMALL;
    PagedParams a;
    a.q = q, a.k = k_pool, a.v = v_pool;
    a.table = table, a.len = len, a.seq = seq, a.n_new = n_new;
    a.share = rows > 0 ? share : nullptr;
    a.out = out, a.lse = lse_out;
    float *w = (float *)((char *)ws + RS_WS_CTRL_BYTES);
    a.cut_o = w, a.row_o = rows ? w + cut * s->D : nullptr;
    float *ml = (float *)((char *)w + align256((cut + rows) * s->D * 4));
    a.cut_ml = ml, a.row_ml = rows ? ml + cut * 2 : nullptr;
    a.B = s->B, a.Hq = s->Hq, a.Hkv = s->Hkv, a.G = s->Hq / s->Hkv;
    a.S = p->S, a.M = p->M, a.N = p->N, a.shift = __builtin_ctz((unsigned)p->P), a.T = T_new, a.groups = kPagedGroups;
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
