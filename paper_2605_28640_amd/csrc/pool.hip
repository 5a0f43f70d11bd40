// Sequences in a pool of pages: who holds which page (reserve, fork, free, compact, share), the copies of a layer's rows that
// follow from it, and the recurrence's append through a table.
//
// A page is free exactly when its reference count is 0, and the lowest numbered free page is always taken first, so there is
// no free list to keep in step: the counts are the only state.  Finding pages is one workgroup's pass over the counts (4 bytes
// a page), in order, with a prefix sum over its threads.  Every call is decided as a whole by that one workgroup before anything is
// written: refused calls change nothing.  What bounds these calls is the trips to memory that follow from one another (list,
// lengths, table, counts: 0.5 us and more each) and the launches themselves, not bytes; so rows of the table are
// written by the deciding workgroup where they are few, and by a second launch over all CUs where they are not.
// Kernel time, us: room for 64 tokens of 64 sequences 6, for 8 questions of up to 384 tokens 7; a release of 4 sequences of 2000 tokens 3, a
// fork 7, their shares 2.4; of 64 with 32700 tokens (two launches each) 7, 10.5, 6.5; compaction of 1000 pages 4.4 + 3.0, of 32768 18 + 5.
#include "check.h"
#include "common.h"

namespace rs {

constexpr int kPoolThreads = 1024;
constexpr int kMaxSeqs = 32768;      // a bit of LDS each
constexpr int kMaxShared = 1024;     // sequences of one page_pool_share call: a thread each
constexpr uint32_t kErrPages = 2u;   // the asynchronous error word of a refused call

// by one thread of a refused call; an expired wait that is on record already says more: outputs of an earlier call are undefined
__device__ __forceinline__ void put_refusal(uint32_t *err)
{
    if (*err == 0u) *err = kErrPages;
}

struct PoolView {
    int32_t *table, *len, *refs;
    int N, S, M, shift;  // shift: log2 of the page size
};

__device__ __forceinline__ int pages_of(int tokens, int shift) { return (int)(((uint32_t)tokens + (1u << shift) - 1) >> shift); }

// what precedes this thread's value among the workgroup's, and (total) their sum; tot: LDS of one word a wave
__device__ __forceinline__ int block_scan_i(int v, int *tot, int &total)
{
    const int wave = threadIdx.x >> 6, inc = wave_scan_i(v);
    if (lane_id() == kWave - 1) tot[wave] = inc;
    __syncthreads();
    int before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kPoolThreads / kWave; ++w) {
        const int x = tot[w];
        if (w < wave) before += x;
        sum += x;
    }
    __syncthreads();
    total = sum;
    return before + inc - v;
}

// The same of values whose sum may pass 32 bits (a call may ask for 2^27 pages 1024 times): 16 bits and the rest of each side by side.  What
// precedes a value is right wherever it fits 32 bits itself.
__device__ __forceinline__ int block_scan_wide(int v, int2 *tot, long &total)
{
    const int wave = threadIdx.x >> 6, low = v & 0xffff, high = v >> 16, l = wave_scan_i(low), h = wave_scan_i(high);
    if (lane_id() == kWave - 1) tot[wave] = make_int2(l, h);
    __syncthreads();
    int2 before = make_int2(l - low, h - high), sum = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < kPoolThreads / kWave; ++w) {
        const int2 x = tot[w];
        if (w < wave) before.x += x.x, before.y += x.y;
        sum.x += x.x, sum.y += x.y;
    }
    __syncthreads();
    total = sum.x + ((long)sum.y << 16);
    return (int)((uint32_t)before.x + ((uint32_t)before.y << 16));
}

// The free pages, ascending, to list, `most` of them; returns how many were found (more perhaps, fewer if there are no more).  Called by
// the whole workgroup.
__device__ __forceinline__ int free_pages(const int32_t *refs, int N, int most, int *tot, int32_t *list)
{
    constexpr int EACH = 16;
    int found = 0;
    for (long base = 0; base < N && found < most; base += kPoolThreads * EACH) {
        const long p0 = base + (long)threadIdx.x * EACH;
        uint32_t mask = 0u;
        if (p0 < N) {
            int r[EACH];
            if (p0 + EACH <= N) {
#pragma unroll
                for (int u = 0; u < EACH / 4; ++u) {
                    const int4 x = *reinterpret_cast<const int4 *>(refs + p0 + 4 * u);
                    r[4 * u] = x.x, r[4 * u + 1] = x.y, r[4 * u + 2] = x.z, r[4 * u + 3] = x.w;
                }
            } else {
#pragma unroll
                for (int u = 0; u < EACH; ++u) r[u] = refs[p0 + u < N ? p0 + u : N - 1];
            }
#pragma unroll
            for (int u = 0; u < EACH; ++u)
                if (p0 + u < N && r[u] <= 0) mask |= 1u << u;
        }
        int total;
        int at = found + block_scan_i(__popc(mask), tot, total);
        for (; mask && at < most; mask &= mask - 1, ++at) list[at] = (int)(p0 + __builtin_ctz(mask));
        found += total;
    }
    return found;
}

// the list entry whose pages include number r: the last i with offs[i] <= r
__device__ __forceinline__ int entry_of(const int32_t *offs, int n, int r)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offs[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// sets a bit of LDS; whether it was set
__device__ __forceinline__ bool seen_before(uint32_t *bits, int s)
{
    return (atomicOr(&bits[s >> 5], 1u << (s & 31)) >> (s & 31)) & 1u;
}

// offs: n words; list: N words
__global__ __launch_bounds__(kPoolThreads) void pool_reserve_kernel(PoolView p, const int32_t *__restrict__ seq, int n,
                                                                    const int32_t *__restrict__ want, int T_new, int32_t *granted,
                                                                    int32_t *offs, int32_t *list, uint32_t *err)
{
    __shared__ uint32_t seen[kMaxSeqs / 32];
    __shared__ int tot[kPoolThreads / kWave];
    __shared__ int2 wide[kPoolThreads / kWave];
    const int tid = threadIdx.x;
    seen[tid] = 0u;
    __syncthreads();
    bool bad = false;
    long needed = 0;
    for (int i0 = 0; i0 < n; i0 += kPoolThreads) {
        const int i = i0 + tid;
        int need = 0;
        if (i < n) {
            const int s = seq[i], t = want ? want[i] : T_new;
            if (s < 0 || s >= p.S || t < 0 || seen_before(seen, s)) {
                bad = true;
            } else {
                const int L = p.len[s];
                if (L < 0 || (long)L + t > (long)p.M << p.shift) bad = true;
                else need = pages_of(L + t, p.shift) - pages_of(L, p.shift);
            }
        }
        // (more than N, or all of it: the same refusal; the wide sum costs every call 0.2 us)
        long total;
        int at;
        if (p.N < (1 << 21) - 1) {
            int sum;
            at = block_scan_i(min(need, p.N + 1), tot, sum);
            total = sum;
        } else {
            at = block_scan_wide(need, wide, total);
        }
        if (i < n) offs[i] = (int)needed + at;  // (no more than N, or nobody looks at it)
        needed += total;
        if (needed > p.N) bad = true;
        if (__syncthreads_or(bad)) break;
    }
    bad = __syncthreads_or(bad);
    const int total = (int)needed;
    if (!bad && total > 0)
        bad = free_pages(p.refs, p.N, total, tot, list) < total;
    __syncthreads();
    if (bad) {
        if (granted)
            for (int i = tid; i < n; i += kPoolThreads) granted[i] = 0;
        if (tid == 0) put_refusal(err);
        return;
    }
    for (int r = tid; r < total; r += kPoolThreads) {
        const int i = entry_of(offs, n, r), s = seq[i], page = list[r];
        p.table[(long)s * p.M + pages_of(p.len[s], p.shift) + (r - offs[i])] = page;
        p.refs[page] = 1;
    }
    __syncthreads();
    for (int i = tid; i < n; i += kPoolThreads) {
        const int t = want ? want[i] : T_new;
        p.len[seq[i]] += t;
        if (granted) granted[i] = t;
    }
}

// a fork's row: the source's first `n` pages, one more reference each; a release's: the same taken back.  By `step` threads from `at` on.
__device__ __forceinline__ void fork_row(const PoolView &p, int src, int dst, int n, int at, int step)
{
    const long s = (long)src * p.M, d = (long)dst * p.M;
    for (int j = at; j < n; j += step) {
        const int page = p.table[s + j];
        p.table[d + j] = page;
        if (page >= 0 && page < p.N) atomicAdd(&p.refs[page], 1);
    }
}
__device__ __forceinline__ void free_row(const PoolView &p, int seq, int n, int at, int step)
{
    const long row = (long)seq * p.M;
    for (int j = at; j < n; j += step) {
        const int page = p.table[row + j];
        p.table[row + j] = -1;
        if (page >= 0 && page < p.N) atomicSub(&p.refs[page], 1);
    }
}
// The rows of n sequences are done by the workgroup that decides, a wave a row at a time, 64 entries a trip, where a wave has at
// most 8 trips to make; else by a launch of their own.  A release, a fork and its copies of n sequences of M pages, us, here / apart:
// 16 of 126 25.8 / 32.5, 32 of 250 26.0 / 30.1, 16 of 501 26.5 / 30.1, 64 of 126 29.9 / 30.1; 16 of 1001 40.6 / 30.2, 64 of 501 51.3 / 38.0.
static bool rows_here(long n, long M) { return (n + 15) / 16 * ((M + 63) / 64) <= 8; }
// Likewise the comparison of neighbours, 256 entries a trip after the two for list and lengths: 16 of 126 28.2 / 32.5, 64 of 126 29.5 / 30.1,
// 4 of 1876 27.3 / 29.8; 64 of 501 41.7 / 38.0.
static bool shares_here(long n, long M) { return (n + 15) / 16 * (2 + (M + 255) / 256) <= 12; }

// full: n words, the pages that entry i takes over from its source (none where the call is refused)
__global__ __launch_bounds__(kPoolThreads) void pool_fork_kernel(PoolView p, const int32_t *__restrict__ src,
                                                                 const int32_t *__restrict__ dst, int n, int2 *pairs, int2 *carry,
                                                                 int32_t *full, int32_t *list, uint32_t *err, bool here)
{
    __shared__ uint32_t seen[kMaxSeqs / 32];
    __shared__ int tot[kPoolThreads / kWave];
    const int tid = threadIdx.x;
    seen[tid] = 0u;
    __syncthreads();
    bool bad = false;
    for (int i = tid; i < n; i += kPoolThreads) {
        const int d = dst[i], s = src[i];
        if (d < 0 || d >= p.S || s < 0 || s >= p.S || seen_before(seen, d) || p.len[d] != 0 || p.len[s] < 0 ||
            p.len[s] > (long)p.M << p.shift)
            bad = true;
    }
    bad = __syncthreads_or(bad);
    for (int i = tid; !bad && i < n; i += kPoolThreads)
        if ((seen[src[i] >> 5] >> (src[i] & 31)) & 1u) bad = true;  // also a destination
    bad = __syncthreads_or(bad);
    int needed = 0;
    for (int i0 = 0; !bad && i0 < n; i0 += kPoolThreads) {  // which of the new pages each entry gets
        const int i = i0 + tid;
        const int need = (i < n && (p.len[src[i]] & ((1 << p.shift) - 1))) ? 1 : 0;
        int total;
        const int at = block_scan_i(need, tot, total);
        if (i < n) full[i] = need ? needed + at : -1;
        needed += total;
    }
    if (!bad && needed > 0)
        bad = free_pages(p.refs, p.N, needed, tot, list) < needed;
    __syncthreads();
    for (int i = tid; i < n; i += kPoolThreads) {
        int2 pr = make_int2(-1, -1), cr = make_int2(-1, -1);
        int whole = 0;
        if (!bad) {
            const int s = src[i], d = dst[i], L = p.len[s], at = full[i];
            whole = L >> p.shift;
            if (at >= 0) {
                pr = make_int2(p.table[(long)s * p.M + whole], list[at]);
                p.refs[pr.y] = 1;
                p.table[(long)d * p.M + whole] = pr.y;
            }
            p.len[d] = L;
            cr = make_int2(s, d);
        }
        full[i] = whole;
        pairs[i] = pr;
        if (carry) carry[i] = cr;
    }
    if (bad && tid == 0) put_refusal(err);
    if (!here || bad) return;
    __syncthreads();
    for (int i = tid >> 6; i < n; i += kPoolThreads / kWave) fork_row(p, src[i], dst[i], full[i], lane_id(), kWave);
}

__global__ __launch_bounds__(256) void pool_fork_rows_kernel(PoolView p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                             const int32_t *__restrict__ full)
{
    const int i = blockIdx.x, n = full[i];
    if (n > 0) fork_row(p, src[i], dst[i], n, blockIdx.y * 256 + threadIdx.x, gridDim.y * 256);
}

// held: n words, the pages that entry i gives up (none where the call is refused)
__global__ __launch_bounds__(kPoolThreads) void pool_free_kernel(PoolView p, const int32_t *__restrict__ seq, int n, int32_t *held,
                                                                 uint32_t *err, bool here)
{
    __shared__ uint32_t seen[kMaxSeqs / 32];
    const int tid = threadIdx.x;
    seen[tid] = 0u;
    __syncthreads();
    bool bad = false;
    for (int i = tid; i < n; i += kPoolThreads) {
        const int s = seq[i];
        if (s < 0 || s >= p.S || seen_before(seen, s) || p.len[s] < 0 || p.len[s] > (long)p.M << p.shift) bad = true;
    }
    bad = __syncthreads_or(bad);
    for (int i = tid; i < n; i += kPoolThreads) {
        held[i] = bad ? 0 : pages_of(p.len[seq[i]], p.shift);
        if (!bad) p.len[seq[i]] = 0;
    }
    if (bad && tid == 0) put_refusal(err);
    if (!here || bad) return;
    __syncthreads();
    for (int i = tid >> 6; i < n; i += kPoolThreads / kWave) free_row(p, seq[i], held[i], lane_id(), kWave);
}

__global__ __launch_bounds__(256) void pool_free_rows_kernel(PoolView p, const int32_t *__restrict__ seq, const int32_t *__restrict__ held)
{
    const int i = blockIdx.x, n = held[i];
    if (n > 0) free_row(p, seq[i], n, blockIdx.y * 256 + threadIdx.x, gridDim.y * 256);
}

// L pages are held: those among them with numbers from L on go, in order, to the free ones below L.  to[page]: where page goes
// (pages from L on that are held); holes, movers: N words; count[0] = L.  Two passes over the counts (how many are held; which are which), every
// thread on 16 of them at a time, and one over the moves.
__global__ __launch_bounds__(kPoolThreads) void pool_compact_kernel(PoolView p, int32_t *to, int32_t *holes, int32_t *movers, int32_t *count,
                                                                    int2 *pairs, int32_t *n_pairs)
{
    constexpr int EACH = 16;
    __shared__ int tot[kPoolThreads / kWave];
    // which of the 16 counts from p0 on are held
    auto held_mask = [&](long p0) __attribute__((always_inline)) -> uint32_t {
        uint32_t mask = 0u;
        if (p0 + EACH <= p.N) {
#pragma unroll
            for (int u = 0; u < EACH / 4; ++u) {
                const int4 x = *reinterpret_cast<const int4 *>(p.refs + p0 + 4 * u);
                mask |= (uint32_t)((x.x > 0) | (x.y > 0) << 1 | (x.z > 0) << 2 | (x.w > 0) << 3) << (4 * u);
            }
        } else {
            for (int u = 0; p0 + u < p.N; ++u) mask |= (uint32_t)(p.refs[p0 + u] > 0) << u;
        }
        return mask;
    };
    int mine = 0, L;
    for (long base = (long)threadIdx.x * EACH; base < p.N; base += kPoolThreads * EACH) mine += __popc(held_mask(base));
    (void)block_scan_i(mine, tot, L);
    int n_holes = 0, n_movers = 0;
    for (long base = 0; base < p.N; base += kPoolThreads * EACH) {
        const long p0 = base + (long)threadIdx.x * EACH;
        const uint32_t held = p0 < p.N ? held_mask(p0) : 0u;
        const long below = p0 >= L ? 0 : min((long)EACH, (long)L - p0), in = p0 >= p.N ? 0 : min((long)EACH, (long)p.N - p0);
        const uint32_t low = (1u << below) - 1u, all = (1u << in) - 1u;
        uint32_t hole = ~held & low & all, mover = held & ~low;
        int total;  // (both numbers in one scan: at most 16384 of each a turn)
        const int at = block_scan_i(__popc(hole) | __popc(mover) << 16, tot, total);
        int h = n_holes + (at & 0xffff), m = n_movers + (at >> 16);
        for (; hole; hole &= hole - 1) holes[h++] = (int)(p0 + __builtin_ctz(hole));
        for (; mover; mover &= mover - 1) movers[m++] = (int)(p0 + __builtin_ctz(mover));
        n_holes += total & 0xffff;
        n_movers += total >> 16;
    }
    __syncthreads();
    constexpr int AHEAD = 4;  // moves on their way together
    for (int r0 = threadIdx.x; r0 < n_holes; r0 += AHEAD * kPoolThreads) {  // (as many movers as holes)
        int from[AHEAD], hole[AHEAD], held[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int r = min(r0 + i * kPoolThreads, n_holes - 1);
            from[i] = movers[r], hole[i] = holes[r];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) held[i] = p.refs[from[i]];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int r = r0 + i * kPoolThreads;
            if (r >= n_holes) break;
            to[from[i]] = hole[i];
            pairs[r] = make_int2(from[i], hole[i]);
            p.refs[hole[i]] = held[i];
            p.refs[from[i]] = 0;
        }
    }
    if (threadIdx.x == 0) {
        count[0] = L;
        n_pairs[0] = n_holes;
    }
}

// the table under the new numbers, and the rest of the list of pairs
__global__ __launch_bounds__(256) void pool_renumber_kernel(PoolView p, const int32_t *__restrict__ to, const int32_t *__restrict__ count,
                                                            int2 *pairs, const int32_t *__restrict__ n_pairs, int room)
{
    const int L = count[0], n = n_pairs[0];
    const long tid = (long)blockIdx.x * 256 + threadIdx.x, all = (long)gridDim.x * 256;
    for (long r = n + tid; r < room; r += all) pairs[r] = make_int2(-1, -1);
    const long cells = (long)p.S * p.M;
    for (long c = tid; c < cells; c += all) {
        const int page = p.table[c];
        if (page >= L && page < p.N && (int)(c % p.M) < pages_of(p.len[c / p.M], p.shift)) p.table[c] = to[page];
    }
}

// leading full pages that sequence i of the list has in common with the one before it, to share[3 i + 1]
__global__ __launch_bounds__(256) void pool_common_kernel(PoolView p, const int32_t *__restrict__ seq, int32_t *share)
{
    const int i = blockIdx.x, tid = threadIdx.x;
    int n = 0;
    if (i > 0) {
        const int a = seq[i - 1], b = seq[i];
        if (a >= 0 && a < p.S && b >= 0 && b < p.S) {
            const int la = p.len[a] >> p.shift, lb = p.len[b] >> p.shift;
            int most = la < lb ? la : lb;
            if (most > p.M) most = p.M;
            const int32_t *ra = p.table + (long)a * p.M, *rb = p.table + (long)b * p.M;
            __shared__ int first;
            for (; n < most; n += 1024) {
                if (tid == 0) first = most;
                __syncthreads();
                int differ = most;
#pragma unroll
                for (int u = 3; u >= 0; --u) {
                    const int j = n + u * 256 + tid;
                    if (j < most && (ra[j] != rb[j] || ra[j] < 0)) differ = j;
                }
                if (differ < most) atomicMin(&first, differ);
                __syncthreads();
                const int f = first;
                __syncthreads();
                if (f < most) {
                    n = f;
                    most = f;
                    break;
                }
            }
            n = most < 0 ? 0 : most;
        }
    }
    if (tid == 0) share[3 * i + 1] = n;
}

// Runs of neighbours with at least `least` pages in common; a run's pages are the fewest that two neighbours in it share.  common: of this
// thread's place of the list with the one before it.
__device__ __forceinline__ void put_runs(int32_t *share, int n, int least, int common)
{
    __shared__ int first[kMaxShared], size[kMaxShared], pages[kMaxShared];
    const int i = threadIdx.x;
    const bool begins = i == 0 || common < least;
    size[i] = 0;
    pages[i] = 0x7fffffff;
    first[i] = begins ? i : 0;
    __syncthreads();
    for (int d = 1; d < n; d <<= 1) {  // running maximum
        const int o = i >= d ? first[i - d] : 0;
        __syncthreads();
        if (o > first[i]) first[i] = o;
        __syncthreads();
    }
    const int f = first[i];
    if (i < n) {
        atomicAdd(&size[f], 1);
        if (!begins) atomicMin(&pages[f], common);
    }
    __syncthreads();
    if (i < n) {
        share[3 * i] = f;
        share[3 * i + 1] = size[f];
        share[3 * i + 2] = size[f] > 1 ? pages[f] : 0;
    }
}
__global__ __launch_bounds__(kMaxShared) void pool_runs_kernel(int32_t *share, int n, int least)
{
    put_runs(share, n, least, (int)threadIdx.x < n ? share[3 * threadIdx.x + 1] : 0);
}
// both at once, for lists of few entries: a wave a pair of neighbours
__global__ __launch_bounds__(kMaxShared) void pool_share_kernel(PoolView p, const int32_t *__restrict__ seq, int32_t *share, int n, int least)
{
    __shared__ int common[kMaxShared];
    if (threadIdx.x == 0) common[0] = 0;
    for (int i = 1 + (threadIdx.x >> 6); i < n; i += kMaxShared / kWave) {
        const int a = seq[i - 1], b = seq[i];
        int same = 0;
        if (a >= 0 && a < p.S && b >= 0 && b < p.S) {
            const int most = min(min(p.len[a] >> p.shift, p.len[b] >> p.shift), p.M);
            const int32_t *ra = p.table + (long)a * p.M, *rb = p.table + (long)b * p.M;
            while (same < most) {
                constexpr int AHEAD = 4;
                int x[AHEAD], y[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int j = min(same + u * kWave + lane_id(), most - 1);
                    x[u] = ra[j], y[u] = rb[j];
                }
                int step = AHEAD * kWave;
#pragma unroll
                for (int u = AHEAD - 1; u >= 0; --u) {
                    const uint64_t differ = __ballot(x[u] != y[u] || x[u] < 0);
                    if (differ) step = u * kWave + __builtin_ctzll(differ);
                }
                if (step < AHEAD * kWave) {
                    same = min(same + step, most);
                    break;
                }
                same = min(same + step, most);
            }
        }
        if (lane_id() == 0) common[i] = max(same, 0);
    }
    __syncthreads();
    put_runs(share, n, least, (int)threadIdx.x < n ? common[threadIdx.x] : 0);
}

struct CopyView {
    const char *k, *v, *meta;
    long head;       // bytes of a KV head's rows
    long meta_head;  // bytes of a KV head's bounds
    int N;
};

// Listed pages of every KV head from one pool to another (or the same).  Nothing but bytes: a page of one head is one run of
// P rows, 2 KB and more.  A workgroup takes (pair, head) after (pair, head).  1.1 GB (7960 pages of 16 tokens, 8 heads of
// 128): 236 us, 4.7 TB/s (a plain copy: 4.9 to 5.1); 64 pages of 64 tokens, 32 heads, 137 MB: 18 us.
__global__ __launch_bounds__(256) void page_copy_kernel(CopyView s, CopyView d, const int2 *__restrict__ pairs, int n,
                                                        const int32_t *__restrict__ n_pairs, int Hkv, int page_bytes, int meta_bytes)
{
    if (n_pairs) n = min(n, max(n_pairs[0], 0));
    const long items = (long)n * Hkv;
    for (long it = blockIdx.x; it < items; it += gridDim.x) {
        const int2 pr = pairs[it / Hkv];
        const long h = it % Hkv;
        if (pr.x < 0 || pr.x >= s.N || pr.y < 0 || pr.y >= d.N) continue;
        const uint4 *ks = reinterpret_cast<const uint4 *>(s.k + h * s.head + (long)pr.x * page_bytes);
        const uint4 *vs = reinterpret_cast<const uint4 *>(s.v + h * s.head + (long)pr.x * page_bytes);
        uint4 *kd = reinterpret_cast<uint4 *>(const_cast<char *>(d.k) + h * d.head + (long)pr.y * page_bytes);
        uint4 *vd = reinterpret_cast<uint4 *>(const_cast<char *>(d.v) + h * d.head + (long)pr.y * page_bytes);
        for (int c = threadIdx.x; c < page_bytes / 16; c += 256) {
            const uint4 a = ks[c], b = vs[c];
            kd[c] = a;
            vd[c] = b;
        }
        if (s.meta) {
            const uint4 *ms = reinterpret_cast<const uint4 *>(s.meta + h * s.meta_head + (long)pr.x * meta_bytes);
            uint4 *md = reinterpret_cast<uint4 *>(const_cast<char *>(d.meta) + h * d.meta_head + (long)pr.y * meta_bytes);
            for (int c = threadIdx.x; c < meta_bytes / 16; c += 256) md[c] = ms[c];
        }
    }
}

__global__ __launch_bounds__(256) void state_copy_kernel(float4 *state_k, float4 *state_v, int S, const int2 *__restrict__ pairs, int row4)
{
    const int2 pr = pairs[blockIdx.x];
    if (pr.x < 0 || pr.x >= S || pr.y < 0 || pr.y >= S) return;
    for (int c = blockIdx.y * 256 + threadIdx.x; c < row4; c += gridDim.y * 256) {
        state_k[(long)pr.y * row4 + c] = state_k[(long)pr.x * row4 + c];
        state_v[(long)pr.y * row4 + c] = state_v[(long)pr.x * row4 + c];
    }
}

struct AppendParams {
    const void *k, *v;
    const float *g;
    float *state_k, *state_v;
    void *k_pool, *v_pool, *meta;
    const int32_t *table, *len, *seq, *n_new;
    int Hkv, S, M, N, shift, T_new;
};

// What an append's workgroup works on: 64 channels of one KV head of one listed sequence, 8 of them a lane, `slice` being the lane's place among those
// that hold the same channels.
template <typename ST, int D>
struct AppendPiece {
    int b, s, L, n;     // list entry, sequence, its tokens, the new ones among them (0: nothing to do)
    int h, c;           // KV head, the lane's first channel
    long state, in;     // of the lane's channels: offset of the carry, of token 0's inputs
    const int32_t *row;
    ST *k_rows, *v_rows, *bounds;

    // the same for the whole workgroup but for c, state, in, and the row pointers
    __device__ __forceinline__ AppendPiece(const AppendParams &a)
    {
        b = blockIdx.x;
        s = a.seq[b];
        const int piece = blockIdx.y;
        h = piece / (D / 64);
        c = piece % (D / 64) * 64 + 8 * (threadIdx.x & 7);
        n = a.n_new ? a.n_new[b] : a.T_new;
        n = n < 0 ? 0 : n > a.T_new ? a.T_new : n;
        int again = 0;  // listed before: nothing is appended twice
        for (int o = threadIdx.x; o < b; o += blockDim.x) again |= a.seq[o] == s;
        again = __syncthreads_or(again);
        L = 0;
        if (again || s < 0 || s >= a.S) {
            n = 0;
            s = 0;
        } else {
            L = a.len[s];
            if (L < n || L > (long)a.M << a.shift) n = 0;
        }
        state = ((long)s * a.Hkv + h) * D + c;
        in = ((long)(b * a.Hkv + h) * a.T_new) * D + c;
        row = a.table + (long)s * a.M;
        const long rows = (long)a.N << a.shift;
        k_rows = (ST *)a.k_pool + (long)h * rows * D + c;
        v_rows = (ST *)a.v_pool + (long)h * rows * D + c;
        bounds = a.meta ? (ST *)a.meta + (long)h * a.N * 2 * D + c : nullptr;
    }
    // the row that holds a position; below 0: the table names no page for it
    __device__ __forceinline__ long row_of(const AppendParams &a, int pos) const
    {
        const int page = row[pos >> a.shift];
        return (page < 0 || page >= a.N) ? -1 : ((long)page << a.shift) + (pos & ((1 << a.shift) - 1));
    }
};

// bounds of rows first, first + STEP, ... below `rows` of a page into lo and hi
template <typename ST, int D, int STEP>
__device__ __forceinline__ void fold_rows(const ST *page, int first, int rows, float (&lo)[8], float (&hi)[8])
{
    constexpr int AHEAD = STEP == 1 ? 16 : 4;  // on their way together
    for (int r = first; r < rows; r += STEP * AHEAD) {
        typename Row8<ST>::raw_t raw[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) raw[i] = Row8<ST>::load_raw(page + (long)(r + STEP * i < rows ? r + STEP * i : r) * D);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float x[8];
            Row8<ST>::unpack(raw[i], x);
#pragma unroll
            for (int j = 0; j < 8; ++j) lo[j] = fminf(lo[j], x[j]), hi[j] = fmaxf(hi[j], x[j]);
        }
    }
}
// over the wave's eight slices, written by the first
template <typename ST, int D>
__device__ __forceinline__ void put_bounds(ST *bounds, int slice, float (&lo)[8], float (&hi)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int m = 8; m < 64; m <<= 1) lo[j] = fminf(lo[j], shfl_xor_f(lo[j], m)), hi[j] = fmaxf(hi[j], shfl_xor_f(hi[j], m));
    if (slice == 0) {
        Row8<ST>::store(bounds, lo);
        Row8<ST>::store(bounds + D, hi);
    }
}

// One token a sequence: s = g s + (1 - g) x in float32, the rounded state to the token's row, its page's bounds from the page's rows so
// far, which need not have been current before.  Nothing but trips to memory: the list, then length and table, then the rows of the
// page, everything else beside them; a wave for 64 channels, its eight slices reading the page's rows side by side.  64
// sequences, 8 heads of 128: 5.3 us (a wave for 128 channels, rows one after the other: 8).
template <typename ST, int D>
__global__ __launch_bounds__(64) void append_token_kernel(const AppendParams a)
{
    const AppendPiece<ST, D> x(a);
    const int slice = threadIdx.x >> 3;
    float sk[8], sv[8], k[8], v[8], g[8];
    Row8<float>::load(a.state_k + x.state, sk);
    Row8<float>::load(a.state_v + x.state, sv);
    Row8<ST>::load((const ST *)a.k + x.in, k);
    Row8<ST>::load((const ST *)a.v + x.in, v);
    Row8<float>::load(a.g + x.in, g);
    if (x.n == 0) return;
    const long row = x.row_of(a, x.L - 1);
    float lo[8], hi[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float om = 1.f - g[j];
        sk[j] = fmaf(g[j], sk[j], om * k[j]);
        sv[j] = fmaf(g[j], sv[j], om * v[j]);
        ST y;
        from_f32(y, sk[j]);
        lo[j] = hi[j] = to_f32(y);
    }
    if (slice == 0) {
        Row8<float>::store(a.state_k + x.state, sk);
        Row8<float>::store(a.state_v + x.state, sv);
        if (row >= 0) {
            Row8<ST>::store(x.k_rows + row * D, sk);
            Row8<ST>::store(x.v_rows + row * D, sv);
        }
    }
    if (x.bounds && row >= 0) {
        const int in_page = (int)(row & ((1 << a.shift) - 1));
        fold_rows<ST, D, 8>(x.k_rows + (row - in_page) * D, slice, in_page, lo, hi);
        put_bounds<ST, D>(x.bounds + (row >> a.shift) * 2 * D, slice, lo, hi);
    }
}

// Several tokens a sequence.  The recurrence is linear, so a run of tokens is (A, S): s -> A s + S, and runs compose: a workgroup takes 32 W tokens at a
// time, 4 a slice; every slice forms its run's (A, S), a scan over the slices (shuffles in a wave, LDS between waves) gives each
// its first state, from which it goes through its 4 tokens as written.  The next tokens' inputs are on their way meanwhile.  Then the bounds
// of the pages touched, from their rows.  8 questions of 150 to 384 tokens, 8 heads of 128: 22 us (token after token 165; with slices of one wave
// only, 32).
template <typename ST, int D, int W>
__global__ __launch_bounds__(64 * W) void append_run_kernel(const AppendParams a)
{
    constexpr int R = 4, CHUNK = 8 * W * R;
    __shared__ float s_run[2][W][3][64];
    const AppendPiece<ST, D> x(a);
    const int slice = (threadIdx.x & 63) >> 3, lane8 = threadIdx.x & 7, wave = threadIdx.x >> 6, n = x.n;
    if (n == 0) return;  // (the whole workgroup)
    struct Inputs {
        typename Row8<ST>::raw_t k[R], v[R];
        typename Row8<float>::raw_t g[R];
        long row[R];
    };
    auto load = [&](int c0, Inputs &in) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int t = c0 + (wave * 8 + slice) * R + r, u = t < n ? t : n - 1;
            in.k[r] = Row8<ST>::load_raw((const ST *)a.k + x.in + (long)u * D);
            in.v[r] = Row8<ST>::load_raw((const ST *)a.v + x.in + (long)u * D);
            in.g[r] = Row8<float>::load_raw(a.g + x.in + (long)u * D);
            in.row[r] = t < n ? x.row_of(a, x.L - n + t) : -1;
        }
    };
    float sk[8], sv[8];  // the carry before the chunk
    Row8<float>::load(a.state_k + x.state, sk);
    Row8<float>::load(a.state_v + x.state, sv);
    Inputs in;
    load(0, in);
#pragma unroll 1
    for (int c0 = 0, buf = 0; c0 < n; c0 += CHUNK, buf ^= 1) {
        const Inputs cur = in;
        if (c0 + CHUNK < n) load(c0 + CHUNK, in);
        const int t0 = c0 + (wave * 8 + slice) * R;
        float A[8], Sk[8], Sv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) A[j] = 1.f, Sk[j] = Sv[j] = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float g[8], k[8], v[8];
            Row8<float>::unpack(cur.g[r], g);
            Row8<ST>::unpack(cur.k[r], k);
            Row8<ST>::unpack(cur.v[r], v);
            if (t0 + r < n) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float om = 1.f - g[j];
                    A[j] *= g[j];
                    Sk[j] = fmaf(g[j], Sk[j], om * k[j]);
                    Sv[j] = fmaf(g[j], Sv[j], om * v[j]);
                }
            }
        }
        // up to and with this slice, within the wave
#pragma unroll
        for (int d = 1; d < 8; d <<= 1)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float pA = __shfl_up(A[j], 8 * d, kWave), pk = __shfl_up(Sk[j], 8 * d, kWave), pv = __shfl_up(Sv[j], 8 * d, kWave);
                if (slice >= d) {
                    Sk[j] = fmaf(A[j], pk, Sk[j]);
                    Sv[j] = fmaf(A[j], pv, Sv[j]);
                    A[j] *= pA;
                }
            }
        if (slice == 7) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s_run[buf][wave][0][lane8 * 8 + j] = A[j];
                s_run[buf][wave][1][lane8 * 8 + j] = Sk[j];
                s_run[buf][wave][2][lane8 * 8 + j] = Sv[j];
            }
        }
        // before this slice, within the wave
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float pA = __shfl_up(A[j], 8, kWave), pk = __shfl_up(Sk[j], 8, kWave), pv = __shfl_up(Sv[j], 8, kWave);
            A[j] = slice ? pA : 1.f;
            Sk[j] = slice ? pk : 0.f;
            Sv[j] = slice ? pv : 0.f;
        }
        __syncthreads();  // (two buffers: the one after next is written only after everyone has passed the next barrier)
        float yk[8], yv[8];
#pragma unroll
        for (int w = 0; w < W; ++w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (w == wave) {
                    yk[j] = fmaf(A[j], sk[j], Sk[j]);
                    yv[j] = fmaf(A[j], sv[j], Sv[j]);
                }
                const float wA = s_run[buf][w][0][lane8 * 8 + j];
                sk[j] = fmaf(wA, sk[j], s_run[buf][w][1][lane8 * 8 + j]);
                sv[j] = fmaf(wA, sv[j], s_run[buf][w][2][lane8 * 8 + j]);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float g[8], k[8], v[8];
            Row8<float>::unpack(cur.g[r], g);
            Row8<ST>::unpack(cur.k[r], k);
            Row8<ST>::unpack(cur.v[r], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float om = 1.f - g[j];
                yk[j] = fmaf(g[j], yk[j], om * k[j]);
                yv[j] = fmaf(g[j], yv[j], om * v[j]);
            }
            if (t0 + r < n) {
                if (cur.row[r] >= 0) {
                    Row8<ST>::store(x.k_rows + cur.row[r] * D, yk);
                    Row8<ST>::store(x.v_rows + cur.row[r] * D, yv);
                }
                if (t0 + r == n - 1) {  // (as this slice has it: the same bits as one token after the other from its first state)
                    Row8<float>::store(a.state_k + x.state, yk);
                    Row8<float>::store(a.state_v + x.state, yv);
                }
            }
        }
    }
    if (!x.bounds) return;
    __syncthreads();  // all rows are written
    const int j0 = (x.L - n) >> a.shift, j1 = (x.L - 1) >> a.shift;
    float lo[8], hi[8];
    // Small pages, many of them: one a slice; larger ones one a wave.  8 runs of 200 tokens, us: pages of 16 22.4 / 27.3, 32 22.9 / 24.1,
    // 64 25.2 / 23.2, 512 53.5 / 28.2.
    if (a.shift <= 5) {
        for (int j = j0 + wave * 8 + slice; j <= j1; j += 8 * W) {
            const int page = x.row[j], rows = min(1 << a.shift, x.L - (j << a.shift));
            if (page < 0 || page >= a.N) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
            fold_rows<ST, D, 1>(x.k_rows + ((long)page << a.shift) * D, 0, rows, lo, hi);
            Row8<ST>::store(x.bounds + (long)page * 2 * D, lo);
            Row8<ST>::store(x.bounds + (long)page * 2 * D + D, hi);
        }
        return;
    }
    for (int j = j0 + wave; j <= j1; j += W) {
        const int page = x.row[j], rows = min(1 << a.shift, x.L - (j << a.shift));
        if (page < 0 || page >= a.N) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
        fold_rows<ST, D, 8>(x.k_rows + ((long)page << a.shift) * D, slice, rows, lo, hi);
        put_bounds<ST, D>(x.bounds + (long)page * 2 * D, slice, lo, hi);
    }
}

// Runs: one wave where the run is at most its 32 tokens at a time or the waves fill the chip without more of them; else four.  One / four, us, with
// the call that makes room: 128 workgroups 32 tokens 14.5 / 14.8, 64 17.8 / 15 to 17, 384 65.7 / 29.8; 512 workgroups 64 22.2 / 25.6, 128
// 34.0 / 29.1; 1024 workgroups 32 19.6 / 40.0, 128 43.4 / 48.8, 384 103 / 112.
template <typename ST, int D>
static void append_launch(const AppendParams &a, int B, hipStream_t stream)
{
    const dim3 grid((unsigned)B, (unsigned)(a.Hkv * (D / 64)));
    const long groups = (long)B * a.Hkv * (D / 64);
    const bool one_wave = a.T_new <= 32 || groups >= 1024 || (groups >= 512 && a.T_new <= 64);
    if (a.T_new == 1) append_token_kernel<ST, D><<<grid, 64, 0, stream>>>(a);
    else if (one_wave) append_run_kernel<ST, D, 1><<<grid, 64, 0, stream>>>(a);
    else append_run_kernel<ST, D, 4><<<grid, 256, 0, stream>>>(a);
}

static PoolView view(const rs_pool *p, int32_t *table, int32_t *len, int32_t *refs)
{
    return PoolView{table, len, refs, p->N, p->S, p->M, __builtin_ctz((unsigned)p->P)};
}

int check_pool(const rs_pool *p)
{
    if (!p || p->N <= 0 || p->S <= 0 || p->M <= 0) return RS_INVALID_ARG;
    if (!page_size_ok(p->P)) return RS_UNSUPPORTED;
    if ((long)p->N * p->P > 0x7fffffffL || (long)p->M * p->P > 0x7fffffffL || p->S > kMaxSeqs) return RS_UNSUPPORTED;
    return RS_OK;
}

// scratch behind the control words: a word for every listed sequence, three for every page, one more
static size_t pool_ws_bytes(const rs_pool *p)
{
    return RS_WS_CTRL_BYTES + align256((size_t)p->S * 4) + 3 * align256((size_t)p->N * 4) + 256;
}

struct PoolScratch {
    uint32_t *err;
    int32_t *seqs, *pages, *pages2, *pages3, *word;
};
static PoolScratch scratch(const rs_pool *p, void *ws)
{
    char *w = (char *)ws + RS_WS_CTRL_BYTES;
    PoolScratch x;
    x.err = (uint32_t *)ws + kCtrlAsyncErr;
    x.seqs = (int32_t *)w;
    x.pages = (int32_t *)(w + align256((size_t)p->S * 4));
    x.pages2 = (int32_t *)((char *)x.pages + align256((size_t)p->N * 4));
    x.pages3 = (int32_t *)((char *)x.pages2 + align256((size_t)p->N * 4));
    x.word = (int32_t *)((char *)x.pages3 + align256((size_t)p->N * 4));
    return x;
}

// what the calls that change a pool ask for in common
static int check_pool_call(const rs_pool *p, const void *table, const void *len, const void *refs, int n, const void *ws, size_t ws_bytes)
{
    const int st = check_pool(p);
    if (st != RS_OK) return st;
    if (!table || !len || !refs || !aligned16(table) || !aligned16(len) || !aligned16(refs)) return RS_INVALID_ARG;
    if (n < 1 || n > p->S) return RS_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < pool_ws_bytes(p)) return RS_WORKSPACE_TOO_SMALL;
    return RS_OK;
}

// workgroups along a table's row: 256 entries each, 64 at most
static unsigned row_groups(const rs_pool *p) { return (unsigned)(p->M >= 64 * 256 ? 64 : (p->M + 255) / 256); }

}  // namespace rs

using namespace rs;

extern "C" {

size_t page_pool_workspace_bytes(const rs_pool *p) { return check_pool(p) == RS_OK ? pool_ws_bytes(p) : 0; }

int32_t page_pool_reserve(const rs_pool *p, int32_t *table, int32_t *len, int32_t *refs, const int32_t *seq, int32_t n, const int32_t *want,
                          int32_t T_new, int32_t *granted, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_pool_call(p, table, len, refs, n, ws, ws_bytes);
    if (st != RS_OK) return st;
    if (!seq || !aligned16(seq) || (want && !aligned16(want)) || (granted && !aligned16(granted)) || T_new < 0) return RS_INVALID_ARG;
    const PoolScratch x = scratch(p, ws);
    pool_reserve_kernel<<<1, kPoolThreads, 0, (hipStream_t)stream>>>(view(p, table, len, refs), seq, n, want, T_new, granted, x.seqs,
                                                                     x.pages, x.err);
    return launch_status();
}

int32_t page_pool_fork(const rs_pool *p, int32_t *table, int32_t *len, int32_t *refs, const int32_t *src, const int32_t *dst, int32_t n,
                       int32_t *pairs_out, int32_t *carry_out, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_pool_call(p, table, len, refs, n, ws, ws_bytes);
    if (st != RS_OK) return st;
    if (!src || !dst || !pairs_out || !aligned16(src) || !aligned16(dst) || !aligned16(pairs_out) || (carry_out && !aligned16(carry_out)))
        return RS_INVALID_ARG;
    const PoolScratch x = scratch(p, ws);
    const PoolView v = view(p, table, len, refs);
    const bool here = rows_here(n, p->M);
    pool_fork_kernel<<<1, kPoolThreads, 0, (hipStream_t)stream>>>(v, src, dst, n, (int2 *)pairs_out, (int2 *)carry_out, x.seqs, x.pages,
                                                                  x.err, here);
    if (!here) pool_fork_rows_kernel<<<dim3((unsigned)n, row_groups(p)), 256, 0, (hipStream_t)stream>>>(v, src, dst, x.seqs);
    return launch_status();
}

int32_t page_pool_free(const rs_pool *p, int32_t *table, int32_t *len, int32_t *refs, const int32_t *seq, int32_t n, void *ws,
                       size_t ws_bytes, void *stream)
{
    const int st = check_pool_call(p, table, len, refs, n, ws, ws_bytes);
    if (st != RS_OK) return st;
    if (!seq || !aligned16(seq)) return RS_INVALID_ARG;
    const PoolScratch x = scratch(p, ws);
    const PoolView v = view(p, table, len, refs);
    const bool here = rows_here(n, p->M);
    pool_free_kernel<<<1, kPoolThreads, 0, (hipStream_t)stream>>>(v, seq, n, x.seqs, x.err, here);
    if (!here) pool_free_rows_kernel<<<dim3((unsigned)n, row_groups(p)), 256, 0, (hipStream_t)stream>>>(v, seq, x.seqs);
    return launch_status();
}

int32_t page_pool_compact(const rs_pool *p, int32_t *table, int32_t *len, int32_t *refs, int32_t *pairs_out, int32_t *n_pairs_out, void *ws,
                          size_t ws_bytes, void *stream)
{
    const int st = check_pool_call(p, table, len, refs, 1, ws, ws_bytes);
    if (st != RS_OK) return st;
    if (!pairs_out || !n_pairs_out || !aligned16(pairs_out) || !aligned16(n_pairs_out)) return RS_INVALID_ARG;
    const PoolScratch x = scratch(p, ws);
    const PoolView v = view(p, table, len, refs);
    pool_compact_kernel<<<1, kPoolThreads, 0, (hipStream_t)stream>>>(v, x.pages, x.pages2, x.pages3, x.word, (int2 *)pairs_out, n_pairs_out);
    const long cells = (long)p->S * p->M;
    const unsigned groups = (unsigned)(cells >= 2048l * 256 ? 2048 : (cells + 255) / 256);
    pool_renumber_kernel<<<groups, 256, 0, (hipStream_t)stream>>>(v, x.pages, x.word, (int2 *)pairs_out, n_pairs_out, p->N > 1 ? p->N / 2 : 1);
    return launch_status();
}

int32_t page_pool_share(const rs_pool *p, const int32_t *table, const int32_t *len, const int32_t *seq, int32_t n, int32_t min_pages,
                        int32_t *share_out, void *stream)
{
    const int st = check_pool(p);
    if (st != RS_OK) return st;
    if (!table || !len || !seq || !share_out || !aligned16(table) || !aligned16(len) || !aligned16(seq) || !aligned16(share_out))
        return RS_INVALID_ARG;
    if (n < 1 || min_pages < 1) return RS_INVALID_ARG;
    if (n > kMaxShared) return RS_UNSUPPORTED;
    const PoolView v = view(p, const_cast<int32_t *>(table), const_cast<int32_t *>(len), nullptr);
    if (shares_here(n, p->M)) {
        pool_share_kernel<<<1, kMaxShared, 0, (hipStream_t)stream>>>(v, seq, share_out, n, min_pages);
        return launch_status();
    }
    pool_common_kernel<<<(unsigned)n, 256, 0, (hipStream_t)stream>>>(v, seq, share_out);
    pool_runs_kernel<<<1, kMaxShared, 0, (hipStream_t)stream>>>(share_out, n, min_pages);
    return launch_status();
}

int32_t page_copy(const rs_shape *s_src, const void *k_src, const void *v_src, const void *meta_src, const rs_shape *s_dst, void *k_dst,
                  void *v_dst, void *meta_dst, const int32_t *pairs, int32_t n, const int32_t *n_pairs, void *stream)
{
    int st = check_rows(s_src, true);
    if (st == RS_OK) st = check_rows(s_dst, true);
    if (st != RS_OK) return st;
    if (s_src->Hkv != s_dst->Hkv || s_src->D != s_dst->D || s_src->P != s_dst->P || s_src->dtype != s_dst->dtype) return RS_INVALID_ARG;
    if (!k_src || !v_src || !k_dst || !v_dst || !pairs || (meta_src == nullptr) != (meta_dst == nullptr)) return RS_INVALID_ARG;
    if (!aligned16(k_src) || !aligned16(v_src) || !aligned16(k_dst) || !aligned16(v_dst) || !aligned16(meta_src) || !aligned16(meta_dst) ||
        !aligned16(pairs) || !aligned16(n_pairs) || n < 1)
        return RS_INVALID_ARG;
    const int row = s_src->D * (int)esize(s_src->dtype);
    auto pool = [row](const rs_shape *s, const void *k, const void *v, const void *meta) {
        return CopyView{(const char *)k, (const char *)v, (const char *)meta, (long)s->Tcap * row, (long)(s->Tcap / s->P) * 2 * row, s->Tcap / s->P};
    };
    const long items = (long)n * s_src->Hkv;
    const unsigned groups = (unsigned)(items < 2048 ? items : 2048);
    page_copy_kernel<<<groups, 256, 0, (hipStream_t)stream>>>(pool(s_src, k_src, v_src, meta_src), pool(s_dst, k_dst, v_dst, meta_dst),
                                                              (const int2 *)pairs, n, n_pairs, s_src->Hkv, s_src->P * row, 2 * row);
    return launch_status();
}

int32_t rat_state_copy(const rs_shape *s, float *state_k, float *state_v, int32_t S, const int32_t *pairs, int32_t n, void *stream)
{
    const int st = check_rows(s, false);
    if (st != RS_OK) return st;
    if (!state_k || !state_v || !pairs || !aligned16(state_k) || !aligned16(state_v) || !aligned16(pairs) || n < 1 || S < 1) return RS_INVALID_ARG;
    const int row4 = s->Hkv * s->D / 4;
    state_copy_kernel<<<dim3((unsigned)n, (unsigned)(row4 < 4096 ? (row4 + 255) / 256 : 16)), 256, 0, (hipStream_t)stream>>>(
        (float4 *)state_k, (float4 *)state_v, S, (const int2 *)pairs, row4);
    return launch_status();
}

int32_t rat_append_paged(const rs_shape *s, const rs_pool *p, const void *k, const void *v, const float *g, float *state_k, float *state_v,
                         void *k_pool, void *v_pool, void *meta, const int32_t *table, const int32_t *len, const int32_t *seq,
                         const int32_t *n_new, int32_t T_new, void *stream)
{
    int st = check_rows(s, true);
    if (st == RS_OK) st = check_pool(p);
    if (st != RS_OK) return st;
    if (p->P != s->P || (long)p->N * p->P != s->Tcap || T_new < 1) return RS_INVALID_ARG;
    if (s->B > kMaxSeqs) return RS_UNSUPPORTED;
    if (!k || !v || !g || !state_k || !state_v || !k_pool || !v_pool || !table || !len || !seq) return RS_INVALID_ARG;
    for (const void *x : {k, v, (const void *)g, (const void *)state_k, (const void *)state_v, (const void *)k_pool, (const void *)v_pool,
                          (const void *)meta, (const void *)table, (const void *)len, (const void *)seq, (const void *)n_new})
        if (!aligned16(x)) return RS_INVALID_ARG;
    const AppendParams a{k, v, g, state_k, state_v, k_pool, v_pool, meta, table, len, seq, n_new, s->Hkv, p->S, p->M, p->N,
                         __builtin_ctz((unsigned)p->P), T_new};
    if (s->dtype == RS_BF16) {
        if (s->D == 128) append_launch<bf16, 128>(a, s->B, (hipStream_t)stream);
        else append_launch<bf16, 64>(a, s->B, (hipStream_t)stream);
    } else {
        if (s->D == 128) append_launch<float, 128>(a, s->B, (hipStream_t)stream);
        else append_launch<float, 64>(a, s->B, (hipStream_t)stream);
    }
    return launch_status();
}

}  // extern "C"
