// A cache in 4 bits: new rows go in, with their pages' bounds, and come back as the values that they stand for.
#include "check.h"
#include "common.h"
#include "kv4.h"

namespace rs {

constexpr int kThreads = 256;
constexpr int kNoPages = 4;  // without bounds: rows go by 16

// eight values of a row
__device__ __forceinline__ void unpack_row(uint32_t codes, float scale, float (&x)[8])
{
    uint32_t p[4];
    kv4_values(codes, scale, p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(p[j] << 16), x[2 * j + 1] = __uint_as_float(p[j] & 0xffff0000u);
}
// the value of the lane m (8, 16 or 32) away
__device__ __forceinline__ float other_rows(float x, int m) { return shfl_xor_f(x, m); }

struct Kv4Params {
    const void *k, *v;  // rows to be stored, T_src of them a head, or nullptr: only the bounds
    const int32_t *len, *n_new;
    uint8_t *k4, *ks, *v4, *vs;
    void *meta;
    long T_src, t_src;
    int Hkv, Tcap, T_new, shift, pages;  // shift: log2 of the page size; pages: that T_new neighbouring rows can lie in
};

// tokens of sequence b, and how many of them are new
__device__ __forceinline__ void sequence(const Kv4Params &a, int b, int &L, int &n)
{
    L = a.len[b];
    n = a.n_new ? a.n_new[b] : a.T_new;
    n = n < 0 ? 0 : n > a.T_new ? a.T_new : n;
    L = L < 0 ? 0 : L > a.Tcap ? a.Tcap : L;
    if (L < n) n = 0;
}

// 16 rows of a page
struct Chunk {
    int page, t0, t1;    // rows t0 .. t1 - 1 of the sequence; t1 <= t0: there are none
    bool begins, ends;   // the page's first, or last, such rows
};

// this lane's 8 channels of a row in 4 bits; x: the channels, then the values that they are stored as
__device__ __forceinline__ void store_row(float (&x)[8], bool real, uint8_t *codes, uint8_t *scales, int c8)
{
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    // over the four lanes of the group
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));  // quad_perm:[1,0,3,2]
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));  // quad_perm:[2,3,0,1]
    const uint32_t byte = kv4_scale_byte(top);
    const uint32_t c = byte == kKv4Nan ? 0u : kv4_codes(x, kv4_scale(byte));
    if (real) {
        reinterpret_cast<uint32_t *>(codes)[c8] = c;
        if ((c8 & 3) == 0) scales[c8 >> 2] = (uint8_t)byte;
    }
    unpack_row(c, kv4_scale(byte), x);
}

template <typename ST>
__device__ __forceinline__ void load_row(const ST *src, bool real, int c8, float (&x)[8])
{
    if (real) Row8<ST>::load(src + 8 * c8, x);
    else
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
}

// Short calls: a workgroup for each (sequence, KV head, page with a new row), D / 8 threads a row.  Nothing but trips to memory, so as many waves as there are
// rows to look at.
template <typename ST, int D>
__global__ __launch_bounds__(kThreads) void kv4_append_short_kernel(const Kv4Params a)
{
    using R = Kv4Row<D>;
    constexpr int CH = D / 8, RPB = kThreads / CH;  // threads a row, rows a turn
    __shared__ float bound[kThreads / kWave][2][D];
    const int bh = blockIdx.y, b = bh / a.Hkv, c8 = threadIdx.x % CH, r0 = threadIdx.x / CH;
    int L, n;
    sequence(a, b, L, n);
    const int P = 1 << a.shift;
    const int first = L - n, page = (first >> a.shift) + blockIdx.x;  // first: the first new token
    if (n == 0 || (page << a.shift) >= L) return;
    const int t0 = page << a.shift, t1 = min(L, t0 + P), from = a.meta ? t0 : max(t0, first);
    float lo[8], hi[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) lo[j] = INFINITY, hi[j] = -INFINITY;
    for (int tb = from; tb < t1; tb += RPB) {
        const int t = tb + r0;
        const bool real = t < t1, fresh = real && t >= first && a.k != nullptr;
        const long row = (long)bh * a.Tcap + t, src = ((long)bh * a.T_src + a.t_src + (t - first)) * D;
        float x[8];
        if (a.k) {
            load_row((const ST *)a.v + src, fresh, c8, x);
            store_row(x, fresh, a.v4 + row * R::CODES, a.vs + row * R::SCALES, c8);
            load_row((const ST *)a.k + src, fresh, c8, x);
            store_row(x, fresh, a.k4 + row * R::CODES, a.ks + row * R::SCALES, c8);
        }
        if (!a.meta || !real) continue;
        if (!fresh) {
            unpack_row(reinterpret_cast<const uint32_t *>(a.k4 + row * R::CODES)[c8], kv4_scale(a.ks[row * R::SCALES + (c8 >> 2)]), x);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) lo[j] = fminf(lo[j], x[j]), hi[j] = fmaxf(hi[j], x[j]);
    }
    if (!a.meta) return;
    // over the rows of a wave, then over the waves
    const int lane = lane_id(), wave = threadIdx.x / kWave;
#pragma unroll
    for (int m = CH; m < kWave; m <<= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j) lo[j] = fminf(lo[j], shfl_xor_f(lo[j], m)), hi[j] = fmaxf(hi[j], shfl_xor_f(hi[j], m));
    if (lane < CH) {
#pragma unroll
        for (int j = 0; j < 8; ++j) bound[wave][0][8 * c8 + j] = lo[j], bound[wave][1][8 * c8 + j] = hi[j];
    }
    __syncthreads();
    ST *const to = (ST *)a.meta + ((long)bh * (a.Tcap >> a.shift) + page) * 2 * D;
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        const int hl = i / D, c = i % D;
        float x = bound[0][hl][c];
        for (int w = 1; w < kThreads / kWave; ++w) x = hl ? fmaxf(x, bound[w][hl][c]) : fminf(x, bound[w][hl][c]);
        from_f32(to[i], x);
    }
}

// Long calls: a wave takes 16 rows of a page at a time, the next ones, if it has more, on their way meanwhile; no other wave has a part in its pages' bounds.
template <typename ST, int D>
__global__ __launch_bounds__(kWave) __attribute__((amdgpu_waves_per_eu(4, 4))) void kv4_append_kernel(const Kv4Params a)
{
    using R = Kv4Row<D>;
    using Raw = typename Row8<ST>::raw_t;
    constexpr int CH = D / 8, RPL = kWave / CH, NG = 16 / RPL;  // lanes a row, rows a load, loads a chunk
    const int lane = lane_id(), c8 = lane % CH, r0 = lane / CH;
    const int bh = blockIdx.y;
    int L, n, at = blockIdx.x;  // at: of the pages with new rows, this wave's
    sequence(a, bh / a.Hkv, L, n);
    const int first = L - n;  // the sequence's first new row
    // the chunk that comes after c; begin: the wave's first
    auto next = [&](Chunk c, bool begin) {
        c.begins = begin || c.ends;
        if (!c.begins) {
            c.t0 += 16;
        } else {
            if (!begin) at += gridDim.x;
            c.page = (first >> a.shift) + at;
            const int row = c.page << a.shift;
            c.t0 = a.meta ? row : max(row, first & ~15);
            c.t1 = n > 0 && at < a.pages ? min(L, row + (1 << a.shift)) : c.t0;
        }
        c.ends = c.t0 + 16 >= c.t1;
        return c;
    };
    auto load = [&](const void *src, const Chunk &c, Raw (&x)[NG]) {
        const int f = max(c.t0, first), n = min(c.t1, c.t0 + 16) - f;  // new rows: f .. f + n - 1
        const LdsSource d = lds_source_sized((const ST *)src + ((long)bh * a.T_src + a.t_src + (f - first)) * D, n > 0 ? n * D * (int)sizeof(ST) : 0);
#pragma unroll
        for (int g = 0; g < NG; ++g) x[g] = load_row8<ST, 2>(d, (uint32_t)(((c.t0 + g * RPL + r0 - f) * D + 8 * c8) * (int)sizeof(ST)));
    };
    Raw kx[NG], vx[NG];
    Chunk c = {};
    c = next(c, true);
    if (c.t1 <= c.t0) return;
    if (a.k) load(a.v, c, vx), load(a.k, c, kx);
    float lo[8], hi[8];
    while (c.t1 > c.t0) {
        const Chunk then = next(c, false);
        if (c.begins) {
#pragma unroll
            for (int j = 0; j < 8; ++j) lo[j] = INFINITY, hi[j] = -INFINITY;
        }
        const bool some_old = c.t0 < first || a.k == nullptr;
        uint32_t old[NG];
        float old_scale[NG];
        if (a.meta && some_old) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const int t = c.t0 + g * RPL + r0;
                const long row = (long)bh * a.Tcap + t;
                const bool is = t < c.t1 && (t < first || a.k == nullptr);
                old[g] = is ? reinterpret_cast<const uint32_t *>(a.k4 + row * R::CODES)[c8] : 0u;
                old_scale[g] = is ? kv4_scale(a.ks[row * R::SCALES + (c8 >> 2)]) : 0.f;
            }
        }
        if (a.k) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const int t = c.t0 + g * RPL + r0;
                const long row = (long)bh * a.Tcap + t;
                float x[8];
                Row8<ST>::unpack(vx[g], x);
                store_row(x, t >= first && t < c.t1, a.v4 + row * R::CODES, a.vs + row * R::SCALES, c8);
            }
            if (then.t1 > then.t0) load(a.v, then, vx);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const int t = c.t0 + g * RPL + r0;
                const long row = (long)bh * a.Tcap + t;
                const bool real = t >= first && t < c.t1;
                float x[8];
                Row8<ST>::unpack(kx[g], x);
                store_row(x, real, a.k4 + row * R::CODES, a.ks + row * R::SCALES, c8);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (real) lo[j] = fminf(lo[j], x[j]), hi[j] = fmaxf(hi[j], x[j]);
            }
            if (then.t1 > then.t0) load(a.k, then, kx);
        }
        if (a.meta) {
            if (some_old) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const int t = c.t0 + g * RPL + r0;
                    float x[8];
                    unpack_row(old[g], old_scale[g], x);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (t < c.t1 && (t < first || a.k == nullptr)) lo[j] = fminf(lo[j], x[j]), hi[j] = fmaxf(hi[j], x[j]);
                }
            }
            if (c.ends) {  // over the wave's rows
#pragma unroll
                for (int m = CH; m < kWave; m <<= 1)
#pragma unroll
                    for (int j = 0; j < 8; ++j) lo[j] = fminf(lo[j], other_rows(lo[j], m)), hi[j] = fmaxf(hi[j], other_rows(hi[j], m));
                ST *const to = (ST *)a.meta + ((long)bh * (a.Tcap >> a.shift) + c.page) * 2 * D + 8 * c8;
                if (r0 == 0) Row8<ST>::store(to, lo);
                if (r0 == 1) Row8<ST>::store(to + D, hi);
            }
        }
        c = then;
    }
}

// 8 channels a thread (32 heads of 32001 tokens of 128 channels, 663 MB: 99 to 121 us)
template <typename ST, int D>
__global__ __launch_bounds__(kThreads) void kv4_fetch_kernel(const uint8_t *__restrict__ k4, const uint8_t *__restrict__ ks,
                                                             const uint8_t *__restrict__ v4, const uint8_t *__restrict__ vs,
                                                             const int32_t *__restrict__ len, long t0, int T, int Tcap, int Hkv, ST *__restrict__ k_out,
                                                             ST *__restrict__ v_out)
{
    using R = Kv4Row<D>;
    constexpr int CH = D / 8, RPB = kThreads / CH;
    const int bh = blockIdx.y, c8 = threadIdx.x % CH;
    const int L = min(len[bh / Hkv], Tcap);
    const long base = t0 < 0 ? (long)L + t0 : t0;
    for (long i = (long)blockIdx.x * RPB + threadIdx.x / CH; i < T; i += (long)gridDim.x * RPB) {
        const long t = base + i;
        if (t < 0 || t >= L) continue;
        const long row = (long)bh * Tcap + t, to = ((long)bh * T + i) * D + 8 * c8;
        const uint32_t kc = reinterpret_cast<const uint32_t *>(k4 + row * R::CODES)[c8], vc = reinterpret_cast<const uint32_t *>(v4 + row * R::CODES)[c8];
        const float kf = kv4_scale(ks[row * R::SCALES + (c8 >> 2)]), vf = kv4_scale(vs[row * R::SCALES + (c8 >> 2)]);
        float x[8];
        unpack_row(kc, kf, x);
        Row8<ST>::store(k_out + to, x);
        unpack_row(vc, vf, x);
        Row8<ST>::store(v_out + to, x);
    }
}

static int append_dispatch(const rs_shape *s, Kv4Params a, hipStream_t stream)
{
    a.Hkv = s->Hkv, a.Tcap = s->Tcap;
    a.pages = (int)(((long)a.T_new + (2l << a.shift) - 2) >> a.shift);
    // Long form against short form, append and read-back of 16 sequences x 8 heads of 128 channels in bfloat16, us: pages of 16, 300 / 600 / 1200 tokens 15.9 / 22.3 / 38.5
    // against 14.5 / 23.7 / 42.8, 32 heads of 32001 tokens 247 against 264; pages of 512, where a wave has 32 turns one after the other, 97 / 112 / 126 against 39 / 54 / 77.
    // (as many waves as there are pages, up to 16 times what fits on the CUs: with 4096 that go on from page to page the 32001 tokens took 270)
    const int BH = s->B * s->Hkv, most = (65536 + BH - 1) / BH;
    const bool stream_form = (long)BH * a.pages >= 4096 && a.T_new >= 1 << a.shift;
    const dim3 grid((unsigned)(!stream_form || a.pages < most ? a.pages : most), (unsigned)BH);
    auto go = [&](auto long_kernel, auto short_kernel) {
        if (stream_form) long_kernel<<<grid, kWave, 0, stream>>>(a);
        else short_kernel<<<grid, kThreads, 0, stream>>>(a);
    };
    if (s->dtype == RS_BF16) {
        if (s->D == 128) go(kv4_append_kernel<bf16, 128>, kv4_append_short_kernel<bf16, 128>);
        else go(kv4_append_kernel<bf16, 64>, kv4_append_short_kernel<bf16, 64>);
    } else {
        if (s->D == 128) go(kv4_append_kernel<float, 128>, kv4_append_short_kernel<float, 128>);
        else go(kv4_append_kernel<float, 64>, kv4_append_short_kernel<float, 64>);
    }
    return launch_status();
}

// what a shape has to be for the calls of a 4-bit cache that take a workgroup's row of the grid for every (sequence, KV head)
static int check_kv4(const rs_shape *s, bool need_page)
{
    const int st = check_rows(s, need_page);
    return st == RS_OK && ((long)s->B * s->Hkv > 65535 || s->Tcap > (1 << 30)) ? RS_UNSUPPORTED : st;
}

template <typename ST, int D>
static int fetch_launch(const rs_shape *s, const uint8_t *k4, const uint8_t *ks, const uint8_t *v4, const uint8_t *vs, const int32_t *len, long t0, int T,
                        void *k_out, void *v_out, hipStream_t stream)
{
    constexpr int RPB = kThreads / (D / 8);
    const long groups = ((long)T + RPB - 1) / RPB;
    kv4_fetch_kernel<ST, D><<<dim3((unsigned)(groups < 4096 ? groups : 4096), (unsigned)(s->B * s->Hkv)), kThreads, 0, stream>>>(
        k4, ks, v4, vs, len, t0, T, s->Tcap, s->Hkv, (ST *)k_out, (ST *)v_out);
    return launch_status();
}

}  // namespace rs

using namespace rs;

extern "C" {

int32_t kv4_append(const rs_shape *s, const void *k, const void *v, int64_t T_src, int64_t t_src, const int32_t *len, const int32_t *n_new,
                   int32_t T_new, uint8_t *k4, uint8_t *k4_scale, uint8_t *v4, uint8_t *v4_scale, void *meta, void *stream)
{
    const int st = check_kv4(s, meta != nullptr);
    if (st != RS_OK) return st;
    if (!k || !v || !len || !k4 || !k4_scale || !v4 || !v4_scale) return RS_INVALID_ARG;
    for (const void *x : {k, v, (const void *)len, (const void *)n_new, (const void *)k4, (const void *)k4_scale, (const void *)v4, (const void *)v4_scale,
                          (const void *)meta})
        if (!aligned16(x)) return RS_INVALID_ARG;
    if (T_new < 1 || T_new > s->Tcap || T_src < 1 || t_src < 0 || t_src > T_src - T_new) return RS_INVALID_ARG;
    Kv4Params a = {};
    a.k = k, a.v = v, a.len = len, a.n_new = n_new, a.k4 = k4, a.ks = k4_scale, a.v4 = v4, a.vs = v4_scale, a.meta = meta;
    a.T_src = T_src, a.t_src = t_src, a.T_new = T_new, a.shift = meta ? __builtin_ctz((unsigned)s->P) : kNoPages;
    return append_dispatch(s, a, (hipStream_t)stream);
}

int32_t kv4_page_meta(const rs_shape *s, const uint8_t *k4, const uint8_t *k4_scale, const int32_t *len, const int32_t *n_new, int32_t T_new, void *meta,
                      void *stream)
{
    const int st = check_kv4(s, true);
    if (st != RS_OK) return st;
    if (!k4 || !k4_scale || !len || !meta) return RS_INVALID_ARG;
    for (const void *x : {(const void *)k4, (const void *)k4_scale, (const void *)len, (const void *)n_new, (const void *)meta})
        if (!aligned16(x)) return RS_INVALID_ARG;
    if (T_new < 1 || T_new > s->Tcap) return RS_INVALID_ARG;
    Kv4Params a = {};
    a.len = len, a.n_new = n_new, a.k4 = const_cast<uint8_t *>(k4), a.ks = const_cast<uint8_t *>(k4_scale), a.meta = meta;
    a.T_new = T_new, a.shift = __builtin_ctz((unsigned)s->P);
    return append_dispatch(s, a, (hipStream_t)stream);
}

int32_t kv4_fetch(const rs_shape *s, const uint8_t *k4, const uint8_t *k4_scale, const uint8_t *v4, const uint8_t *v4_scale, const int32_t *len,
                  int64_t t0, int32_t T, void *k_out, void *v_out, void *stream)
{
    const int st = check_kv4(s, false);
    if (st != RS_OK) return st;
    if (!k4 || !k4_scale || !v4 || !v4_scale || !len || !k_out || !v_out) return RS_INVALID_ARG;
    for (const void *x : {(const void *)k4, (const void *)k4_scale, (const void *)v4, (const void *)v4_scale, (const void *)len, (const void *)k_out,
                          (const void *)v_out})
        if (!aligned16(x)) return RS_INVALID_ARG;
    if (T < 1 || t0 < -(int64_t)s->Tcap || t0 >= s->Tcap) return RS_INVALID_ARG;
    hipStream_t q = (hipStream_t)stream;
    if (s->dtype == RS_BF16)
        return s->D == 128 ? fetch_launch<bf16, 128>(s, k4, k4_scale, v4, v4_scale, len, t0, T, k_out, v_out, q)
                           : fetch_launch<bf16, 64>(s, k4, k4_scale, v4, v4_scale, len, t0, T, k_out, v_out, q);
    return s->D == 128 ? fetch_launch<float, 128>(s, k4, k4_scale, v4, v4_scale, len, t0, T, k_out, v_out, q)
                       : fetch_launch<float, 64>(s, k4, k4_scale, v4, v4_scale, len, t0, T, k_out, v_out, q);
}

}  // extern "C"
