// A cache in 4 bits: new rows go in, with their pages' bounds, and come back as the values that they stand for.
#include "check.h"
#include "common.h"
#include "kv4.h"

namespace rs {

constexpr int kThreads = 256;
constexpr int kNoPages = 4;  // without bounds: rows go by 16

struct Kv4Params {
    const void *k, *v;  // rows to be stored, T_src of them a head, or nullptr: only the bounds
    const int32_t *len, *n_new;
    uint8_t *k4, *ks, *v4, *vs;
    void *meta;
    long T_src, t_src;
    int Hkv, Tcap, T_new, shift;  // shift: log2 of the page size
};

// tokens of sequence b, and how many of them are new
__device__ __forceinline__ void sequence(const Kv4Params &a, int b, int &L, int &n)
{
    L = a.len[b];
    n = a.n_new ? a.n_new[b] : a.T_new;
    n = n < 0 ? 0 : n > a.T_new ? a.T_new : n;
    if (L > a.Tcap) L = a.Tcap;
    if (L < n) n = 0;  // (a length below 0 among them)
}

// this lane's 8 channels of a row, in 4 bits; returned as the values that they stand for
template <typename ST, int D>
__device__ __forceinline__ void store_row(const ST *src, uint8_t *codes, uint8_t *scales, int c8, bool real, float (&x)[8])
{
    if (real) Row8<ST>::load(src + 8 * c8, x);
    else
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    // over the four lanes of the group
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));  // quad_perm:[1,0,3,2]
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));  // quad_perm:[2,3,0,1]
    const uint32_t byte = kv4_scale_byte(top);
    const float scale = kv4_scale(byte);
    const uint32_t c = byte == kKv4Nan ? 0u : kv4_codes(x, scale);
    if (real) {
        reinterpret_cast<uint32_t *>(codes)[c8] = c;
        if ((c8 & 3) == 0) scales[c8 >> 2] = (uint8_t)byte;
    }
    uint32_t p[4];
    kv4_values(c, scale, p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(p[j] << 16), x[2 * j + 1] = __uint_as_float(p[j] & 0xffff0000u);
}

// A workgroup for each (sequence, KV head, page with a new row): D / 8 threads a row.
template <typename ST, int D>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(const Kv4Params a)
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
            store_row<ST, D>((const ST *)a.v + src, a.v4 + row * R::CODES, a.vs + row * R::SCALES, c8, fresh, x);
            store_row<ST, D>((const ST *)a.k + src, a.k4 + row * R::CODES, a.ks + row * R::SCALES, c8, fresh, x);
        }
        if (!a.meta || !real) continue;
        if (!fresh) {
            uint32_t p[4];
            kv4_values(reinterpret_cast<const uint32_t *>(a.k4 + row * R::CODES)[c8], kv4_scale(a.ks[row * R::SCALES + (c8 >> 2)]), p);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(p[j] << 16), x[2 * j + 1] = __uint_as_float(p[j] & 0xffff0000u);
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

// 8 channels a thread
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
        uint32_t p[4];
        float x[8];
        kv4_values(kc, kf, p);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(p[j] << 16), x[2 * j + 1] = __uint_as_float(p[j] & 0xffff0000u);
        Row8<ST>::store(k_out + to, x);
        kv4_values(vc, vf, p);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(p[j] << 16), x[2 * j + 1] = __uint_as_float(p[j] & 0xffff0000u);
        Row8<ST>::store(v_out + to, x);
    }
}

template <typename ST, int D>
static int append_launch(const Kv4Params &a, int BH, hipStream_t stream)
{
    const int P = 1 << a.shift, pages = (int)(((long)a.T_new + 2l * P - 2) / P);  // that T_new neighbouring rows can lie in
    kv4_append_kernel<ST, D><<<dim3((unsigned)pages, (unsigned)BH), kThreads, 0, stream>>>(a);
    return launch_status();
}

static int append_dispatch(const rs_shape *s, const Kv4Params &a, hipStream_t stream)
{
    const int BH = s->B * s->Hkv;
    if (s->dtype == RS_BF16) return s->D == 128 ? append_launch<bf16, 128>(a, BH, stream) : append_launch<bf16, 64>(a, BH, stream);
    return s->D == 128 ? append_launch<float, 128>(a, BH, stream) : append_launch<float, 64>(a, BH, stream);
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
    return append_dispatch(s, Kv4Params{k, v, len, n_new, k4, k4_scale, v4, v4_scale, meta, T_src, t_src, s->Hkv, s->Tcap, T_new,
                                        meta ? __builtin_ctz((unsigned)s->P) : kNoPages}, (hipStream_t)stream);
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
    return append_dispatch(s, Kv4Params{nullptr, nullptr, len, n_new, const_cast<uint8_t *>(k4), const_cast<uint8_t *>(k4_scale), nullptr, nullptr, meta,
                                        0, 0, s->Hkv, s->Tcap, T_new, __builtin_ctz((unsigned)s->P)}, (hipStream_t)stream);
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
