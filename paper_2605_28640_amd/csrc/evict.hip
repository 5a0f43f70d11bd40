// Sequences that have outgrown their budget: of every KV head's rows those with the largest tallies stay, and the first and the newest ones.
// Which rows stay is decided by a workgroup for each (sequence, KV head): the n_keep-th largest key by a radix search (11, 11 and 10 bits), ties
// to the lower row; where only a few rows go, as in a decode step, by taking the smallest that often.
// Rows do not have to lie in the order of their positions, so only those kept rows move that lie behind the first n_keep, to the places
// of the dropped ones before it: the i-th of them to the i-th hole.  Sources and destinations are apart, so they move in any order: a few by the
// deciding workgroup, many by a second launch on all CUs.
#include "check.h"
#include "common.h"

namespace rs {

constexpr int kThreads = 1024;
constexpr int kFewGo = 8;       // up to so many dropped rows are looked for one by one
constexpr int kMovedHere = 64;  // up to so many rows are moved by the workgroup that chose them
constexpr int kTurn = 256;      // rows that a wave looks at together
constexpr int kBins = 2048, kCopies = 2;
constexpr int kMostHeld = 34816;  // keys that fit in LDS beside the bins
constexpr uint32_t kStays = 0xffffffffu;  // the key of a row that stays whatever its tally (+inf: 0xff800000)

struct MovedRows {
    char *rows[4];  // K and V, or their codes and scale bytes
    int bytes[4];   // a row
    int n;
};

struct EvictParams {
    float *tally;
    int32_t *pos, *mark, *len;
    int4 *count;         // [B Hkv] rows that the second launch moves; rows whose position is on record, tokens seen up to them
    uint32_t *arrived;   // [B] workgroups of a sequence that are done; zero before and after
    int32_t *from, *to;  // [B Hkv, most] rows that move, and where
    uint32_t *keys;      // [B Hkv, key_row], of caches with more rows than LDS holds
    long most, key_row;
    MovedRows moved;
    int Hkv, Tcap, keep, first, recent, slack;
};

// pieces of U bytes
template <typename U>
__device__ __forceinline__ void move_rows(char *rows, int bytes, const int32_t *from, const int32_t *to, int n, long at, long step)
{
    const int per = bytes / (int)sizeof(U);
    for (long i = at; i < (long)n * per; i += step) {
        const int r = (int)(i / per), c = (int)(i - (long)r * per);
        reinterpret_cast<U *>(rows + (long)to[r] * bytes)[c] = reinterpret_cast<const U *>(rows + (long)from[r] * bytes)[c];
    }
}
__device__ __forceinline__ void move_all(const EvictParams &a, int bh, int known, int before, const int32_t *from, const int32_t *to, int n, long at, long step)
{
    float *const tally = a.tally + (long)bh * a.Tcap;
    int32_t *const pos = a.pos + (long)bh * a.Tcap;
    for (long i = at; i < n; i += step) {
        const int f = from[i], t = to[i];
        tally[t] = tally[f];
        pos[t] = f < known ? pos[f] : before + (f - known);
    }
    for (int i = 0; i < a.moved.n; ++i) {
        char *rows = a.moved.rows[i] + (long)bh * a.Tcap * a.moved.bytes[i];
        if (a.moved.bytes[i] % 16 == 0) move_rows<uint4>(rows, a.moved.bytes[i], from, to, n, at, step);
        else move_rows<uint16_t>(rows, a.moved.bytes[i], from, to, n, at, step);
    }
}

// sum over the wave, in every lane
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan_i(x), kWave - 1); }

// inclusive sums over the waves: `before` gets what the waves before this one hold, the return value is all.  lds: not in use by an earlier call
template <int WAVES>
__device__ __forceinline__ int wave_offsets(int x, int *lds, int &before)
{
    const int wave = threadIdx.x / kWave;
    if (lane_id() == 0) lds[wave] = x;
    __syncthreads();
    int sum = 0;
    before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) before = sum;
        sum += lds[w];
    }
    return sum;
}

template <typename F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, F f)
{
#pragma unroll
    for (int m = kWave / 2; m >= 1; m >>= 1) x = f(x, (uint32_t)__shfl_xor((int)x, m, kWave));
    return x;
}

// (Positions that repeat, of which more than `keep` rows could have to stay: the first `keep` of those do.)
// Keys are looked at several times: from LDS, where HELD of them fit, or (0) from memory.  A wave takes neighbouring rows, 256 a turn, four neighbours
// a thread.  (Keys in registers instead, 32 a thread, made loops of 32 copies and spilled: 36 us for 16384 rows of 32 heads, 57 from memory.)
template <int HELD, int THREADS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictParams a)
{
    constexpr int WAVES = THREADS / kWave, EACH = kBins / THREADS;  // bins a thread
    __shared__ __attribute__((aligned(16))) uint32_t held[HELD > 0 ? HELD : 4];
    __shared__ __attribute__((aligned(16))) uint32_t hist[kBins][kCopies];
    __shared__ int lds[3][WAVES];
    __shared__ __attribute__((aligned(16))) int4 counts[WAVES];
    __shared__ int found[2];
    __shared__ uint32_t least[2][WAVES][2];
    __shared__ int32_t few_from[kMovedHere], few_to[kMovedHere];
    const int bh = blockIdx.x, b = bh / a.Hkv, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int L = min(a.len[b], a.Tcap);
    const int known = max(0, min(a.mark[2 * b], L)), before = a.mark[2 * b + 1];
    const bool over = L > a.keep && L - a.keep > a.slack;
    if (!over) {
        if (threadIdx.x == 0) a.count[bh] = make_int4(0, 0, 0, 0);
        return;
    }
    const int total = before + L - known, n_go = L - a.keep;
    float *const tally = a.tally + (long)bh * a.Tcap;
    int32_t *const pos = a.pos + (long)bh * a.Tcap;
    uint32_t *const keys = HELD > 0 ? held : a.keys + bh * a.key_row;
    auto position = [&](int t) { return t < known ? pos[t] : before + (t - known); };
    const int turns = (L + WAVES * kTurn - 1) / (WAVES * kTurn), from = min(L, wave * turns * kTurn), to = min(L, from + turns * kTurn);
    // ---- the keys; rows up to a whole turn that there are not stay ----
    constexpr int AHEAD = 16;  // loads of a thread on their way together
    for (int t0 = from; t0 < to; t0 += AHEAD * kWave) {
        float x[AHEAD];
        int p[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i * kWave + lane;
            x[i] = t < to ? tally[t] : 0.f;
            p[i] = t < to ? position(t) : 0;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i * kWave + lane;
            const uint32_t k = t >= to || p[i] < a.first || p[i] >= total - a.recent ? kStays : x[i] != x[i] ? 0u : float_to_key(x[i]);
            if (t0 + i / 4 * kTurn < to) keys[t] = k;
        }
    }
    for (int i = threadIdx.x; i < kBins * kCopies; i += THREADS) (&hist[0][0])[i] = 0;
    __syncthreads();
    auto load4 = [&](int t0) { return *reinterpret_cast<const uint4 *>(keys + t0 + 4 * lane); };
    int n_movers;
    if (HELD > 0 && n_go <= kFewGo) {
        int gone[kFewGo];
#pragma unroll
        for (int i = 0; i < kFewGo; ++i) {
            gone[i] = 0x7fffffff;
            if (i >= n_go) continue;
            // the smallest key, and of equal ones the last row (there is one unless positions repeat, see below)
            uint32_t k = kStays;
            int at = -1;
            for (int t0 = from; t0 < to; t0 += kTurn) {
                const uint4 x = load4(t0);
                const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (v[c] <= k && v[c] != kStays) k = v[c], at = t0 + 4 * lane + c;
            }
            const uint32_t wk = wave_reduce(k, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
            const uint32_t wt = wave_reduce(k == wk ? (uint32_t)(at + 1) : 0u, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
            if (lane == 0) least[i & 1][wave][0] = wk, least[i & 1][wave][1] = wt;
            __syncthreads();
            uint32_t gk = kStays, gt = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const uint32_t x = least[i & 1][w][0], t = least[i & 1][w][1];
                if (x < gk || (x == gk && t > gt)) gk = x, gt = t;
            }
            if (gt > 0) gone[i] = (int)gt - 1;
            if (gone[i] >= from && gone[i] < to) keys[gone[i]] = kStays;  // (its own wave, which alone looks at it)
        }
        // every thread has all of them: thread i works out the i-th hole and the i-th mover
        n_movers = 0;
#pragma unroll
        for (int i = 0; i < kFewGo; ++i) n_movers += gone[i] < a.keep;
        if (threadIdx.x < kFewGo) {
#pragma unroll
            for (int i = 0; i < kFewGo; ++i) {  // hole: as many smaller ones as this thread's number
                int rank = 0;
#pragma unroll
                for (int j = 0; j < kFewGo; ++j) rank += gone[j] < gone[i];
                if (gone[i] < a.keep && rank == (int)threadIdx.x) few_to[threadIdx.x] = gone[i];
            }
            const int t = a.keep + (int)threadIdx.x;
            int rank = 0;
            bool stays = t < L;
#pragma unroll
            for (int j = 0; j < kFewGo; ++j) stays &= gone[j] != t, rank += gone[j] >= a.keep && gone[j] < t;
            if (stays) few_from[(int)threadIdx.x - rank] = t;
        }
        for (int t = known + threadIdx.x; t < a.keep; t += THREADS) {
            bool hole = false;
#pragma unroll
            for (int i = 0; i < kFewGo; ++i) hole |= gone[i] == t;
            if (!hole) pos[t] = before + (t - known);
        }
    } else {
        // ---- the keep-th largest key ----
        uint32_t prefix = 0;
        const int no_rows = kTurn - 1 - (L + kTurn - 1) % kTurn;
        int left = a.keep + no_rows;  // of the keys that begin with the prefix, the left-th largest (rows that there are not count in)
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int t0 = from; t0 < to; t0 += kTurn) {
                const uint4 x = load4(t0);
                const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (pass == 0 || (v[c] >> (shift + bits)) == (prefix >> (shift + bits))) atomicAdd(&hist[(v[c] >> shift) & ((1u << bits) - 1u)][lane % kCopies], 1u);
            }
            __syncthreads();
            // the bins from the top, EACH a thread, which leaves them empty for the next pass
            int n[EACH], sum = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                uint32_t *const bin = hist[kBins - 1 - (EACH * threadIdx.x + i)];
                n[i] = 0;
#pragma unroll
                for (int c = 0; c < kCopies; ++c) n[i] += (int)bin[c], bin[c] = 0;
                sum += n[i];
            }
            const int incl = wave_scan_i(sum);
            int above;
            wave_offsets<WAVES>(__builtin_amdgcn_readlane(incl, kWave - 1), lds[pass], above);
            above += incl - sum;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (above < left && above + n[i] >= left) found[0] = kBins - 1 - (EACH * threadIdx.x + i), found[1] = left - above;
                above += n[i];
            }
            __syncthreads();
            prefix |= (uint32_t)found[0] << shift;
            left = found[1];
        }
        if (prefix == kStays) left -= no_rows;  // no rows but those that have to stay
        // Keys above the prefix stay, and of those equal to it the first `left`.  How many there are of both, before row `keep` and behind it, wave by wave:
        // where each wave's holes (rows before `keep` that go) and movers (rows behind it that stay) come.
        int4 mine = make_int4(0, 0, 0, 0);
        for (int t0 = from; t0 < to; t0 += kTurn) {
            const uint4 x = load4(t0);
            const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int t = t0 + 4 * lane + c, above = v[c] > prefix, same = v[c] == prefix;
                if (t < a.keep) mine.x += above, mine.y += same;
                else if (t < L) mine.z += above, mine.w += same;
            }
        }
        mine = make_int4(wave_total(mine.x), wave_total(mine.y), wave_total(mine.z), wave_total(mine.w));
        if (lane == 0) counts[wave] = mine;
        __syncthreads();
        int eq = 0, holes = 0, movers = 0, e = 0;
        n_movers = 0;
        for (int w = 0; w < WAVES; ++w) {
            const int4 c = counts[w];
            if (w == wave) eq = e, movers = n_movers;
            const int f = min(L, w * turns * kTurn), before_keep = max(0, min(a.keep, min(L, f + turns * kTurn)) - f);
            const int kept0 = max(0, min(left - e, c.y)), kept1 = max(0, min(left - e - c.y, c.w));
            if (w < wave) holes += before_keep - c.x - kept0;
            n_movers += c.z + kept1;
            e += c.y + c.w;
        }
        const bool fit = n_movers <= kMovedHere;
        int32_t *const hole = fit ? few_to : a.to + bh * a.most, *const mover = fit ? few_from : a.from + bh * a.most;
        for (int t0 = from; t0 < to; t0 += kTurn) {
            const uint4 x = load4(t0);
            const uint32_t v[4] = {x.x, x.y, x.z, x.w};
            const int t = t0 + 4 * lane;
            uint32_t stays = 0;  // four bits
#pragma unroll
            for (int c = 0; c < 4; ++c) stays |= (v[c] > prefix ? 1u : 0u) << c;
            if (mine.y + mine.w > 0) {  // the wave has rows that are equal to the last one that stays
                uint32_t same = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) same |= (v[c] == prefix && t + c < L ? 1u : 0u) << c;
                const int incl = wave_scan_i(__popc(same));
                int rank = eq + incl - __popc(same);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if ((same >> c) & 1) {
                        if (rank < left) stays |= 1u << c;
                        ++rank;
                    }
                eq += __builtin_amdgcn_readlane(incl, kWave - 1);
            }
            const uint32_t real = L - t >= 4 ? 15u : L > t ? (1u << (L - t)) - 1u : 0u, front = a.keep - t >= 4 ? 15u : a.keep > t ? (1u << (a.keep - t)) - 1u : 0u;
            auto put = [&](uint32_t which, int32_t *list, int &at) {
                const int incl = wave_scan_i(__popc(which));
                int i = at + incl - __popc(which);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if ((which >> c) & 1) list[i++] = t + c;
                at += __builtin_amdgcn_readlane(incl, kWave - 1);
            };
            if (t0 < a.keep) put(~stays & real & front, hole, holes);
            if (t0 + kTurn > a.keep) put(stays & real & ~front, mover, movers);
            if (t0 < a.keep && t0 + kTurn > known) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (((stays & front) >> c) & 1 && t + c >= known) pos[t + c] = before + (t + c - known);
            }
        }
    }
    __syncthreads();
    const bool here = n_movers <= kMovedHere;
    if (here) move_all(a, bh, known, before, few_from, few_to, n_movers, threadIdx.x, THREADS);
    if (threadIdx.x == 0) {
        a.count[bh] = make_int4(here ? 0 : n_movers, known, before, 0);
        // the last of the sequence's workgroups, all of which have read its length by now
        if (atomicAdd(a.arrived + b, 1u) == (uint32_t)a.Hkv - 1u) {
            a.arrived[b] = 0u;
            a.len[b] = a.keep;
            a.mark[2 * b] = a.keep;
            a.mark[2 * b + 1] = total;
        }
    }
}

__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams a)
{
    const int bh = blockIdx.y;
    const int4 c = a.count[bh];
    move_all(a, bh, c.y, c.z, a.from + bh * a.most, a.to + bh * a.most, c.x, (long)blockIdx.x * blockDim.x + threadIdx.x, (long)gridDim.x * blockDim.x);
}

struct EvictLayout {
    size_t count, from, to, keys, total;
    long most, key_row;
};
static EvictLayout evict_layout(const rs_shape *s, int keep)
{
    EvictLayout x;
    const size_t BH = (size_t)s->B * s->Hkv;
    x.most = keep < s->Tcap - keep ? keep : s->Tcap - keep;
    x.key_row = s->Tcap > kMostHeld ? ((long)s->Tcap + kTurn - 1) / kTurn * kTurn : 0;
    x.count = RS_WS_CTRL_BYTES;
    x.from = x.count + align256(BH * 16);
    x.to = x.from + align256(BH * (size_t)x.most * 4);
    x.keys = x.to + align256(BH * (size_t)x.most * 4);
    x.total = x.keys + BH * (size_t)x.key_row * 4;
    return x;
}

static int check_evict(const rs_shape *s, int keep)
{
    const int st = check_rows(s, false);
    if (st != RS_OK) return st;
    if (keep < 1 || keep > s->Tcap) return RS_INVALID_ARG;
    return (long)s->B * s->Hkv > 65535 || s->B > 2 * kMaxUnits || s->Tcap > (1 << 30) ? RS_UNSUPPORTED : RS_OK;
}

static int evict_run(const rs_shape *s, const MovedRows &m, float *tally, int32_t *pos, int32_t *mark, int32_t *len, int keep, int first, int recent,
                     int slack, void *ws, size_t ws_bytes, hipStream_t stream)
{
    for (const void *x : {(const void *)tally, (const void *)pos, (const void *)mark, (const void *)len})
        if (!x || !aligned16(x)) return RS_INVALID_ARG;
    for (int i = 0; i < m.n; ++i)
        if (!m.rows[i] || !aligned16(m.rows[i])) return RS_INVALID_ARG;
    if (first < 0 || recent < 0 || slack < 0 || (long)first + recent > keep) return RS_INVALID_ARG;
    const EvictLayout x = evict_layout(s, keep);
    if (!ws || !aligned16(ws) || ws_bytes < x.total) return RS_WORKSPACE_TOO_SMALL;
    char *const w = (char *)ws;
    const int BH = s->B * s->Hkv;
    const EvictParams a{tally, pos, mark, len, (int4 *)(w + x.count), (uint32_t *)ws + kCtrlUnit0, (int32_t *)(w + x.from), (int32_t *)(w + x.to), (uint32_t *)(w + x.keys),
                        x.most, x.key_row, m, s->Hkv, s->Tcap, keep, first, recent, slack};
    // Short caches of more heads than compute units: four waves a head, of which a compute unit holds six at once (46 registers, 26 KB of LDS; only one with 16 waves).  1504 heads of 119 rows, 72 kept:
    // 33 us, 57 with 16 waves; 500 rows less one: 24, 41; 2000, half kept: 211, 230.  With fewer heads the 16 waves win: 256 heads of 2000 rows 39 to 41.
    if (s->Tcap <= 2304 && BH > 256) evict_select_kernel<2304, 256><<<BH, 256, 0, stream>>>(a);
    else if (s->Tcap <= 8704) evict_select_kernel<8704, kThreads><<<BH, kThreads, 0, stream>>>(a);
    else if (s->Tcap <= 17408) evict_select_kernel<17408, kThreads><<<BH, kThreads, 0, stream>>>(a);
    else if (s->Tcap <= kMostHeld) evict_select_kernel<kMostHeld, kThreads><<<BH, kThreads, 0, stream>>>(a);
    else evict_select_kernel<0, kThreads><<<BH, kThreads, 0, stream>>>(a);
    if (x.most <= kMovedHere) return launch_status();  // no call on this cache has more to move
    // about 2048 workgroups, and not more than have 4 KB to move
    long parts = (2048 + BH - 1) / BH, need = (x.most * m.bytes[0] + 4095) / 4096;
    if (parts > need) parts = need < 1 ? 1 : need;
    evict_move_kernel<<<dim3((unsigned)parts, (unsigned)BH), 256, 0, stream>>>(a);
    return launch_status();
}

}  // namespace rs

using namespace rs;

extern "C" {

size_t cache_evict_workspace_bytes(const rs_shape *s, int32_t n_keep) { return check_evict(s, n_keep) == RS_OK ? evict_layout(s, n_keep).total : 0; }

int32_t cache_evict(const rs_shape *s, void *k_cache, void *v_cache, float *tally, int32_t *pos, int32_t *mark, int32_t *len, int32_t n_keep, int32_t n_first,
                    int32_t n_recent, int32_t n_slack, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_evict(s, n_keep);
    if (st != RS_OK) return st;
    MovedRows m = {};
    const int row = s->D * (int)esize(s->dtype);
    m.n = 2;
    m.rows[0] = (char *)k_cache, m.rows[1] = (char *)v_cache;
    m.bytes[0] = m.bytes[1] = row;
    return evict_run(s, m, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws, ws_bytes, (hipStream_t)stream);
}

int32_t kv4_evict(const rs_shape *s, uint8_t *k4, uint8_t *k4_scale, uint8_t *v4, uint8_t *v4_scale, float *tally, int32_t *pos, int32_t *mark, int32_t *len,
                  int32_t n_keep, int32_t n_first, int32_t n_recent, int32_t n_slack, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_evict(s, n_keep);
    if (st != RS_OK) return st;
    MovedRows m = {};
    m.n = 4;
    m.rows[0] = (char *)k4, m.rows[1] = (char *)v4, m.rows[2] = (char *)k4_scale, m.rows[3] = (char *)v4_scale;
    m.bytes[0] = m.bytes[1] = s->D / 2;
    m.bytes[2] = m.bytes[3] = s->D / 32;
    return evict_run(s, m, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws, ws_bytes, (hipStream_t)stream);
}

}  // extern "C"
