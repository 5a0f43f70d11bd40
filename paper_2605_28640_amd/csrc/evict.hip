// Sequences that have outgrown their budget: of every KV head's rows those with the largest tallies stay, and the first and the newest ones.
// Which rows stay is decided by a workgroup for each (sequence, KV head): the n_keep-th largest key by a radix search, ties to the lower row.
// Rows do not have to lie in the order of their positions, so only those kept rows move that lie behind the first n_keep, to the places
// of the dropped ones before it: the i-th of them to the i-th hole.  Sources and destinations are apart, so they move in any order (a second
// launch, all CUs).
#include "check.h"
#include "common.h"

namespace rs {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;

struct EvictParams {
    float *tally;
    int32_t *pos, *mark, *len;
    int32_t *state, *count;  // [B, 2] length afterwards (-1: as it is), tokens seen; [B Hkv] rows that move
    int2 *pairs;             // [B Hkv, most] (from, to)
    uint32_t *keys;          // [B Hkv, Tcap]
    long most;
    int Hkv, Tcap, keep, first, recent, slack;
};

// inclusive prefix sums of one number a wave: *before gets those of the waves before this one, the return value is the sum of all
__device__ __forceinline__ int wave_offsets(int x, int *lds, int &before)
{
    const int wave = threadIdx.x / kWave;
    __syncthreads();
    if (lane_id() == 0) lds[wave] = x;
    __syncthreads();
    int sum = 0;
    before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = sum;
        sum += lds[w];
    }
    return sum;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(const EvictParams a)
{
    constexpr int COPIES = 16;
    __shared__ uint32_t hist[256][COPIES];
    __shared__ int lds[kWaves];
    __shared__ int found[2];
    const int bh = blockIdx.x, b = bh / a.Hkv, lane = lane_id(), wave = threadIdx.x / kWave;
    const int L = min(a.len[b], a.Tcap);
    const int known = max(0, min(a.mark[2 * b], L)), before = a.mark[2 * b + 1];
    const bool over = L > a.keep && L - a.keep > a.slack;
    const int total = before + L - known;
    if (threadIdx.x == 0) {
        if (bh == b * a.Hkv) a.state[2 * b] = over ? a.keep : -1, a.state[2 * b + 1] = total;
        if (!over) a.count[bh] = 0;
    }
    if (!over) return;
    float *const tally = a.tally + (long)bh * a.Tcap;
    int32_t *const pos = a.pos + (long)bh * a.Tcap;
    uint32_t *const keys = a.keys + (long)bh * a.Tcap;
    auto position = [&](int t) { return t < known ? pos[t] : before + (t - known); };
    // a wave's rows: a multiple of 64 of them
    const int each = (L + kThreads - 1) / kThreads * kWave, from = min(L, wave * each), to = min(L, from + each);
    for (int t = from + lane; t < to; t += kWave) {
        const int p = position(t);
        const float x = tally[t];
        keys[t] = p < a.first || p >= total - a.recent ? 0xffffffffu : x != x ? 0u : float_to_key(x);
    }
    // ---- the keep-th largest key ----
    uint32_t prefix = 0;
    int left = a.keep;  // of the keys that begin with the prefix, the left-th largest
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256 * COPIES; i += kThreads) (&hist[0][0])[i] = 0;
        __syncthreads();
        for (int t = from + lane; t < to; t += kWave) {
            const uint32_t k = keys[t];
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u][lane % COPIES], 1u);
        }
        __syncthreads();
        if (wave < 4) {  // digit 255 - threadIdx.x: those above it come first
            const int d = 255 - threadIdx.x;
            int n = 0;
#pragma unroll
            for (int c = 0; c < COPIES; ++c) n += (int)hist[d][(c + d) % COPIES];
            int incl = wave_scan_i(n);
            if (lane == kWave - 1) lds[wave] = incl;
            hist[d][0] = (uint32_t)incl;
            hist[d][1] = (uint32_t)n;
        }
        __syncthreads();
        if (wave < 4) {
            const int d = 255 - threadIdx.x, n = (int)hist[d][1];
            int incl = (int)hist[d][0];
            for (int w = 0; w < wave; ++w) incl += lds[w];
            if (incl >= left && incl - n < left) found[0] = d, found[1] = left - (incl - n);
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        left = found[1];
    }
    // keys above the prefix stay, and of those equal to it the first `left`
    int mine = 0;
    for (int t0 = from; t0 < to; t0 += kWave) mine += __popcll(__ballot(t0 + lane < to && keys[min(t0 + lane, L - 1)] == prefix));
    int equal;
    wave_offsets(mine, lds, equal);
    // rows before `keep` that go, and rows behind it that stay: a wave's numbers, then their places
    int n_holes = 0, n_movers = 0, holes, movers;
    for (int round = 0; round < 2; ++round) {
        int eq = equal, h = 0, m = 0;
        for (int t0 = from; t0 < to; t0 += kWave) {
            const int t = t0 + lane;
            const bool real = t < to;
            const uint32_t k = real ? keys[t] : 0u;
            const uint64_t same = __ballot(real && k == prefix);
            const int rank = eq + __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
            const bool stays = real && (k > prefix || (k == prefix && rank < left));
            const bool hole = real && t < a.keep && !stays, mover = t >= a.keep && stays;
            const uint64_t hm = __ballot(hole), mm = __ballot(mover);
            if (round) {
                if (hole) a.pairs[bh * a.most + holes + h + __builtin_amdgcn_mbcnt_hi((uint32_t)(hm >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hm, 0u))].y = t;
                if (mover) a.pairs[bh * a.most + movers + m + __builtin_amdgcn_mbcnt_hi((uint32_t)(mm >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mm, 0u))].x = t;
                if (stays && t < a.keep && t >= known) pos[t] = position(t);
            }
            eq += __popcll(same);
            h += __popcll(hm);
            m += __popcll(mm);
        }
        if (!round) {
            n_holes = wave_offsets(h, lds, holes);
            n_movers = wave_offsets(m, lds, movers);
        }
    }
    (void)n_holes;  // as many as movers
    if (threadIdx.x == 0) a.count[bh] = n_movers;
    __syncthreads();
    for (int i = threadIdx.x; i < n_movers; i += kThreads) {
        const int2 p = a.pairs[bh * a.most + i];
        tally[p.y] = tally[p.x];
        pos[p.y] = position(p.x);
    }
}

struct MoveParams {
    char *rows[4];   // K and V, or their codes and scale bytes
    int row_bytes[4];
    int n;
    const int2 *pairs;
    const int32_t *count, *state;
    int32_t *len, *mark;
    long most;
    int Hkv, Tcap, keep;
};

// pieces of U bytes
template <typename U>
__device__ __forceinline__ void move_rows(char *rows, int bytes, const int2 *pairs, int n, int part, int parts)
{
    const int per = bytes / (int)sizeof(U);
    for (long i = (long)part * blockDim.x + threadIdx.x; i < (long)n * per; i += (long)parts * blockDim.x) {
        const int2 p = pairs[i / per];
        const int c = (int)(i % per);
        reinterpret_cast<U *>(rows + (long)p.y * bytes)[c] = reinterpret_cast<const U *>(rows + (long)p.x * bytes)[c];
    }
}

__global__ __launch_bounds__(256) void evict_move_kernel(const MoveParams a)
{
    const int bh = blockIdx.y, b = bh / a.Hkv;
    if (blockIdx.x == 0 && threadIdx.x == 0 && bh == b * a.Hkv && a.state[2 * b] >= 0) {
        a.len[b] = a.keep;
        a.mark[2 * b] = a.keep;
        a.mark[2 * b + 1] = a.state[2 * b + 1];
    }
    const int n = a.count[bh];
    const int2 *pairs = a.pairs + bh * a.most;
    for (int i = 0; i < a.n; ++i) {
        char *rows = a.rows[i] + (long)bh * a.Tcap * a.row_bytes[i];
        if (a.row_bytes[i] % 16 == 0) move_rows<uint4>(rows, a.row_bytes[i], pairs, n, blockIdx.x, gridDim.x);
        else move_rows<uint16_t>(rows, a.row_bytes[i], pairs, n, blockIdx.x, gridDim.x);
    }
}

struct EvictLayout {
    size_t state, count, pairs, keys, total;
    long most;
};
static EvictLayout evict_layout(const rs_shape *s, int keep)
{
    EvictLayout x;
    const size_t BH = (size_t)s->B * s->Hkv;
    x.most = keep < s->Tcap - keep ? keep : s->Tcap - keep;
    x.state = RS_WS_CTRL_BYTES;
    x.count = x.state + align256((size_t)s->B * 8);
    x.pairs = x.count + align256(BH * 4);
    x.keys = x.pairs + align256(BH * (size_t)x.most * 8);
    x.total = x.keys + align256(BH * (size_t)s->Tcap * 4);
    return x;
}

static int check_evict(const rs_shape *s, int keep)
{
    const int st = check_rows(s, false);
    if (st != RS_OK) return st;
    if (keep < 1 || keep > s->Tcap) return RS_INVALID_ARG;
    return (long)s->B * s->Hkv > 65535 || s->Tcap > (1 << 30) ? RS_UNSUPPORTED : RS_OK;
}

static int evict_run(const rs_shape *s, MoveParams m, float *tally, int32_t *pos, int32_t *mark, int32_t *len, int keep, int first, int recent, int slack,
                     void *ws, size_t ws_bytes, hipStream_t stream)
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
    const EvictParams a{tally, pos, mark, len, (int32_t *)(w + x.state), (int32_t *)(w + x.count), (int2 *)(w + x.pairs), (uint32_t *)(w + x.keys), x.most,
                        s->Hkv, s->Tcap, keep, first, recent, slack};
    evict_select_kernel<<<BH, kThreads, 0, stream>>>(a);
    m.pairs = a.pairs, m.count = a.count, m.state = a.state, m.len = len, m.mark = mark, m.most = x.most;
    m.Hkv = s->Hkv, m.Tcap = s->Tcap, m.keep = keep;
    // about 2048 workgroups, and not more than have 4 KB to move
    long parts = (2048 + BH - 1) / BH, need = (x.most * m.row_bytes[0] + 4095) / 4096;
    if (parts > need) parts = need < 1 ? 1 : need;
    evict_move_kernel<<<dim3((unsigned)parts, (unsigned)BH), 256, 0, stream>>>(m);
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
    MoveParams m = {};
    const int row = s->D * (int)esize(s->dtype);
    m.n = 2;
    m.rows[0] = (char *)k_cache, m.rows[1] = (char *)v_cache;
    m.row_bytes[0] = m.row_bytes[1] = row;
    return evict_run(s, m, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws, ws_bytes, (hipStream_t)stream);
}

int32_t kv4_evict(const rs_shape *s, uint8_t *k4, uint8_t *k4_scale, uint8_t *v4, uint8_t *v4_scale, float *tally, int32_t *pos, int32_t *mark, int32_t *len,
                  int32_t n_keep, int32_t n_first, int32_t n_recent, int32_t n_slack, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_evict(s, n_keep);
    if (st != RS_OK) return st;
    MoveParams m = {};
    m.n = 4;
    m.rows[0] = (char *)k4, m.rows[1] = (char *)v4, m.rows[2] = (char *)k4_scale, m.rows[3] = (char *)v4_scale;
    m.row_bytes[0] = m.row_bytes[1] = s->D / 2;
    m.row_bytes[2] = m.row_bytes[3] = s->D / 32;
    return evict_run(s, m, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws, ws_bytes, (hipStream_t)stream);
}

}  // extern "C"
