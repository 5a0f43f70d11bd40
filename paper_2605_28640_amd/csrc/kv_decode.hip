// One token's dense attention over caches of sequences of different lengths, with a tally of the weight that every row has had, and the
// same over whole or listed pages of a 4-bit cache.
//   z_t = scale q . k_t,  m = max z,  l = sum e^(z_t - m),  out = sum e^(z_t - m) v_t / l,  tally_t += sum over a KV head's queries of e^(z_t - m) / l
// Work: a tile is a KV head's (listed pages of a query head: the query head's) up to 16 queries of one sequence; its tokens, in units of a wave's step (4 bits: 64,
// bfloat16: 32, float32: 16), lie on a
// line, tile after tile, sequence after sequence.  The line is divided evenly among the waves, whatever the lengths, which every workgroup reads
// for itself.  A wave goes through its share without a pause: the next step's rows and, where a tile begins, its queries are on their way before
// the present step is done.  A tile that lies in one share is done with it; one that is cut leaves records, which a second launch joins in their order
// on the line (the four waves of a workgroup that is all inside one tile leave one).  So the order of every sum follows from the lengths alone.
// The tally needs the weights' sum over all tokens, so the scores (float32) go to the workspace and the second launch turns them into weights.
// Caches that are a few steps long take a workgroup a tile and one launch.
#include "check.h"
#include "common.h"
#include "kv4.h"

namespace rs {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kQ = 16;         // queries of a tile, at most
constexpr int kUnit = 64;      // tokens of the largest unit
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kMaxB = 1024;
constexpr float kSlack = 8.f;  // the reference point of a softmax moves when the maximum has grown by more (base-2 exponent): weights stay below 2^8

struct DecodeParams {
    const void *q, *k, *v;        // k, v: rows, or codes
    const uint8_t *ks, *vs;       // scale bytes
    const int32_t *len, *idx;
    void *out;
    float *lse, *tally;
    float *rec_o, *rec_ml, *lse2, *z;  // records [2 a wave, rows, D], [.., 2]; base-2 log-sum-exps [B, Hq]; scores [B, Hq, z_row]
    int *start;                   // [B + 1] units of the sequences before
    int B, Hq, Hkv, H, G, RT, D;  // H: heads with tiles of their own, G queries each, in RT tiles
    int Tcap, K, shift, list_units, z_row, groups, rows, fresh, unit;  // unit: tokens of one, a wave's step
    bool three;  // workgroups to a CU
    float scale;
};

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
// over the wave, in every lane: within rows of 16 by rotations, then over the four rows
__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, dpp_f<0x128>(x));
    x = fmaxf(x, dpp_f<0x124>(x));
    x = fmaxf(x, dpp_f<0x122>(x));
    return quad_max(fmaxf(x, dpp_f<0x121>(x)));
}
__device__ __forceinline__ float wave_sum(float x) { return quad_sum(group_sum<16>(x)); }
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int length_of(const DecodeParams &a, int b)
{
    const int n = a.len[b];
    return n < 0 ? 0 : n > a.Tcap ? a.Tcap : n;
}
__device__ __forceinline__ int units_of(const DecodeParams &a, int n) { return a.idx ? (n > 0 ? a.list_units : 0) : (n + a.unit - 1) / a.unit; }

// a b / c for whole numbers whose product is below 2^53: the rounded quotient is a whole number only where the exact one is (another one is at least 1 / c away
// from it), so cutting it off is exact.  (Divisions of 64-bit integers, which a wave begins with several of, made every call 20 us longer.)
__device__ __forceinline__ int product_over(int a, double b, double c) { return (int)((double)a * b / c); }

// The line's shares, one a wave.  Of the workgroups on a CU the one that came first gets most of what the CU asks of memory: with equal shares of 4 x 32 heads
// of 64K tokens the first 256 workgroups were done after 122 us, the others after 143 and 168.  So where three fit on a CU and every wave has
// some steps to go, the shares are weighted (that call 185 -> 173 us, its 256 listed pages a head 26.9 -> 25.5; two or four to a CU: no gain).
constexpr int kTurn = 256 * kWaves;                  // waves of a workgroup on every CU
constexpr int kWeight[3] = {54, 43, 31};             // they add up to 128
struct LineShares {
    int total, n;
    bool weighted;

    LineShares() = default;
    __device__ __forceinline__ LineShares(int sum, int heads, int groups, bool three)
    {
        total = sum * heads;
        n = total < groups * kWaves ? total : groups * kWaves;
        weighted = three && total >= 8 * kTurn;  // (the smallest has a unit or more: none is empty)
    }
    __device__ __forceinline__ int begin(int i) const
    {
        if (!weighted) return product_over(i, total, n);
        const int at = i <= kTurn ? kWeight[0] * i
                                  : i <= 2 * kTurn ? kWeight[0] * kTurn + kWeight[1] * (i - kTurn)
                                                   : (kWeight[0] + kWeight[1]) * kTurn + kWeight[2] * (i - 2 * kTurn);
        return (int)((long)at * total / (128 * kTurn));
    }
    __device__ __forceinline__ int of(int unit) const  // whose a unit is
    {
        if (!weighted) return (int)((((double)unit + 1) * n - 1) / total);
        const int at = (int)((((double)unit + 1) * (128 * kTurn) - 1) / total);
        if (at < kWeight[0] * kTurn) return at / kWeight[0];
        if (at < (kWeight[0] + kWeight[1]) * kTurn) return kTurn + (at - kWeight[0] * kTurn) / kWeight[1];
        return 2 * kTurn + (at - (kWeight[0] + kWeight[1]) * kTurn) / kWeight[2];
    }
};

struct LineTile {
    int b, h, rt, s0, s1, L;  // sequence, head, 16 queries of it, its units on the line; tokens of the sequence
};

// Where the sequences' units begin.  Up to 64 sequences: a lane of every wave each, nothing but the lengths' trip to memory; more: in LDS.
struct LinePlan {
    int first, units, len;  // of sequence lane_id()
    const int *start;       // [B + 1] in LDS, or nullptr
    int sum;

    __device__ __forceinline__ void make(const DecodeParams &a, int *lds, int *wave_tot)
    {
        if (a.B <= kWave) {
            const int b = lane_id();
            len = b < a.B ? length_of(a, b) : 0;
            units = units_of(a, len);
            const int incl = wave_scan_i(units);
            first = incl - units;
            sum = __builtin_amdgcn_readlane(incl, kWave - 1);
            start = nullptr;
            return;
        }
        constexpr int EACH = kMaxB / kThreads;
        const int t = threadIdx.x, lane = lane_id(), wave = t / kWave;
        int x[EACH], all = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int b = t * EACH + i;
            x[i] = b < a.B ? units_of(a, length_of(a, b)) : 0;
            all += x[i];
        }
        const int incl = wave_scan_i(all);
        if (lane == kWave - 1) wave_tot[wave] = incl;
        __syncthreads();
        int at = incl - all;
        for (int w = 0; w < wave; ++w) at += wave_tot[w];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int b = t * EACH + i;
            if (b <= a.B) lds[b] = at;
            at += x[i];
        }
        if (t == kThreads - 1 && a.B == kMaxB) lds[kMaxB] = at;
        __syncthreads();
        start = lds;
        sum = scalar(lds[a.B]);
    }
    __device__ __forceinline__ int begin(int b) const { return start ? start[b] : __shfl(first, b, kWave); }  // (b < B)
    __device__ __forceinline__ LineTile find(const DecodeParams &a, int unit) const
    {
        const int HR = a.H * a.RT;
        LineTile w;
        int from, n;  // the last sequence that does not begin behind the unit
        if (!start) {
            w.b = 63 - __builtin_clzll(__ballot(lane_id() < a.B && first * HR <= unit));
            from = __builtin_amdgcn_readlane(first, w.b);
            n = __builtin_amdgcn_readlane(units, w.b);
            w.L = __builtin_amdgcn_readlane(len, w.b);
        } else {
            int lo = 0, hi = a.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (scalar(start[mid]) * HR <= unit) lo = mid;
                else hi = mid;
            }
            w.b = lo;
            from = scalar(start[lo]);
            n = scalar(start[lo + 1]) - from;
            w.L = scalar(length_of(a, lo));
        }
        const int hr = (unit - from * HR) / n;
        w.h = a.RT == 1 ? hr : hr / a.RT;
        w.rt = a.RT == 1 ? 0 : hr - w.h * a.RT;
        w.s0 = from * HR + hr * n;
        w.s1 = w.s0 + n;
        return w;
    }
};

// the token row that a query's first 16 tokens of a unit begin at, and how many of them there are
template <int NH>
struct StepWhere {
    int at[NH], valid[NH];
};

// The weights of eight tokens as three bfloat16 operands whose sum they are, all 24 bits of them.  A term is what the ones before leave,
// cut off after 8 bits: a mask, a difference, and a byte permute for two.  (With weights rounded to one bfloat16 term 24 ragged sequences take 38.6 us instead of
// 39.4 and 256 listed pages a head 24.7 instead of 25.6, 64K tokens 178 instead of 174; but a result then has an error of its own besides its last rounding.)
// ROWS: the values may be infinite (in 4 bits they are not), and 0 times that is NaN: a term for which nothing is left is 2^-30 of the weight instead, two of them
// a 32nd of its last bit (of weights below 2^-96 nothing is left of that either).
template <bool ROWS>
__device__ __forceinline__ void split3(const f32x4 &p0, const f32x4 &p1, bf16x8 (&out)[3])
{
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = i < 2 ? p0[2 * i] : p1[2 * i - 4], b = i < 2 ? p0[2 * i + 1] : p1[2 * i - 3];
        const float least_a = a * 0x1p-30f, least_b = b * 0x1p-30f;
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            if (ROWS && n > 0) a = fmaxf(a, least_a), b = fmaxf(b, least_b);
            const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
            w[n][i] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);  // the upper halves, a's below
            if (n < 2) a -= __uint_as_float(ua & 0xffff0000u), b -= __uint_as_float(ub & 0xffff0000u);
        }
    }
#pragma unroll
    for (int n = 0; n < 3; ++n) out[n] = __builtin_bit_cast(bf16x8, make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]));
}

// ---- the rows of a step: 16 NH tokens ------------------------------------------------------------------------------------
// Lane (l16, lg) = (lane % 16, lane / 16) takes token l16 of every 16 as the K operand, and query l16.  V goes through a tile in LDS: 32 bfloat16
// rows (float32: 16), 16-byte chunks permuted so that the transpose reads of the product touch every bank once.
template <bool FOUR, typename ST, int D>
struct StepRows;

// 4 bits: a lane's part of a row is D / 8 neighbouring bytes, D / 4 channels of one group: one load, one scale.  The queries' channels follow.
template <typename ST, int D>
struct StepRows<true, ST, D> {
    static constexpr int NH = 4, NK = D / 32, TERMS = sizeof(ST) == 2 ? 1 : 3, ROW = 2 * D, CODES = D / 2, SCALES = D / 32;
    uint32_t kc[NH][NK], vc[NH][NK], kf[NH], vf[NH];
    bf16x8 qf[TERMS][NK];
    int lane, l16, lg;

    __device__ __forceinline__ static int swizzle(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }
    __device__ __forceinline__ void load_q(const ST *q, bool real)
    {
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            float x[8];
            Row8<ST>::load(q + lg * (D / 4) + kk * 8, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float rest = real ? x[j] : 0.f;
#pragma unroll
                for (int n = 0; n < TERMS; ++n) {  // float32 as the sum of three bfloat16 numbers, all of its 24 bits: each cuts off (rounding up could make an infinity)
                    const uint32_t u = __float_as_uint(rest);
                    qf[n][kk][j] = __builtin_bit_cast(__bf16, (unsigned short)(u >> 16));
                    rest = (u & 0x7fffffffu) == 0x7f800000u ? 0.f : rest - __uint_as_float(u & 0xffff0000u);  // (nothing is left of an infinity)
                }
            }
        }
    }
    template <int N>
    __device__ __forceinline__ static void load_codes(LdsSource src, uint32_t at, uint32_t (&c)[N])
    {
        if constexpr (N == 4) {
            const auto x = __builtin_amdgcn_raw_buffer_load_b128(src, at, 0, 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = (uint32_t)x[i];
        } else {
            const auto x = __builtin_amdgcn_raw_buffer_load_b64(src, at, 0, 2);
            c[0] = (uint32_t)x[0], c[1] = (uint32_t)x[1];
        }
    }
    __device__ __forceinline__ void load_k(const DecodeParams &a, long base, const StepWhere<NH> &x)
    {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const long row = base + x.at[h];
            load_codes(lds_source_sized((const uint8_t *)a.k + row * CODES, x.valid[h] * CODES), (uint32_t)(l16 * CODES + lg * (CODES / 4)), kc[h]);
            kf[h] = __builtin_amdgcn_raw_buffer_load_b8(lds_source_sized(a.ks + row * SCALES, x.valid[h] * SCALES),
                                                        (uint32_t)(l16 * SCALES + (D == 128 ? lg : lg >> 1)), 0, 0);
        }
    }
    __device__ __forceinline__ void load_v(const DecodeParams &a, long base, const StepWhere<NH> &x)
    {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const long row = base + x.at[h];
            load_codes(lds_source_sized((const uint8_t *)a.v + row * CODES, x.valid[h] * CODES), (uint32_t)(lane * (CODES / 4)), vc[h]);
            vf[h] = __builtin_amdgcn_raw_buffer_load_b8(lds_source_sized(a.vs + row * SCALES, x.valid[h] * SCALES),
                                                        (uint32_t)((lane >> 2) * SCALES + (D == 128 ? lane & 3 : (lane & 3) >> 1)), 0, 0);
        }
    }
    // S^T = K Q^T of 16 tokens: tokens 4 lg .. 4 lg + 3 of query l16
    __device__ __forceinline__ f32x4 scores(int h) const
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        const float f = kv4_scale(kf[h] & 255u);
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            uint32_t p[4];
            kv4_values(kc[h][kk], f, p);
            const bf16x8 k = __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3]));
#pragma unroll
            for (int n = 0; n < TERMS; ++n) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[n][kk], s, 0, 0, 0);
        }
        return s;
    }
    // O^T += V^T P^T; p: the weights of all 16 NH tokens
    __device__ __forceinline__ void values(char *tile, const f32x4 (&p)[NH], f32x4 (&o)[D / 16])
    {
#pragma unroll
        for (int half = 0; half < NH / 2; ++half) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = 16 * h + (lane >> 2);
                const float f = kv4_scale(vf[2 * half + h] & 255u);
#pragma unroll
                for (int c = 0; c < NK; ++c) {
                    uint32_t w[4];
                    kv4_values(vc[2 * half + h][c], f, w);
                    *reinterpret_cast<uint4 *>(tile + row * ROW + (((lane & 3) * NK + c) ^ swizzle(row)) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            product32<D, false>(tile, p[2 * half], p[2 * half + 1], o, l16, lg);
        }
    }
    // 32 tokens, whose values are in the tile
    template <int DD, bool ROWS>
    __device__ __forceinline__ static void product32(const char *tile, const f32x4 &p0, const f32x4 &p1, f32x4 (&o)[DD / 16], int l16, int lg)
    {
        bf16x8 pf[3];
        split3<ROWS>(p0, p1, pf);
        const int r = 4 * lg + (l16 >> 2);
        const uint32_t at = (uint32_t)(r * 2 * DD + ((((l16 & 3) >> 1) ^ swizzle(r)) * 16) + 8 * (l16 & 1));
#pragma unroll
        for (int dt = 0; dt < DD / 16; ++dt) {
            union {
                s16x4 h[2];
                bf16x8 f;
            } x;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                x.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(tile + (at ^ (uint32_t)(32 * dt)) + h * 16 * 2 * DD));
#pragma unroll
            for (int n = 0; n < 3; ++n) o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.f, pf[n], o[dt], 0, 0, 0);
        }
    }
};

// bfloat16 and float32 rows: 16-byte operands at chunk 4 kk + lg of a row
template <typename ST, int D>
struct StepRows<false, ST, D> {
    static constexpr bool BF = sizeof(ST) == 2;
    static constexpr int NH = BF ? 2 : 1, ROW = D * (int)sizeof(ST), NK = ROW / 64, CR = ROW / 16, RW = 64 / CR, NL = 16 / RW;
    f32x4 kx[NH][NK], vx[NH][NL], qf[NK];
    int lane, l16, lg;

    __device__ __forceinline__ static int swizzle(int row)
    {
        if (!BF) return 4 * ((row >> 2) & 3);
        return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3);
    }
    __device__ __forceinline__ void load_q(const ST *q, bool real)
    {
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const char *>(q) + 64 * kk + 16 * lg);
            qf[kk] = real ? x : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void load_k(const DecodeParams &a, long base, const StepWhere<NH> &x)
    {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const LdsSource src = lds_source_sized((const char *)a.k + (base + x.at[h]) * ROW, x.valid[h] * ROW);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk)
                kx[h][kk] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (uint32_t)(l16 * ROW + lg * 16 + 64 * kk), 0, 2));
        }
    }
    __device__ __forceinline__ void load_v(const DecodeParams &a, long base, const StepWhere<NH> &x)
    {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const LdsSource src = lds_source_sized((const char *)a.v + (base + x.at[h]) * ROW, x.valid[h] * ROW);
#pragma unroll
            for (int i = 0; i < NL; ++i) vx[h][i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (uint32_t)(lane * 16 + 1024 * i), 0, 2));
        }
    }
    __device__ __forceinline__ f32x4 scores(int h) const
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            if constexpr (BF) {
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[h][kk]), __builtin_bit_cast(bf16x8, qf[kk]), s, 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[h][kk][j], qf[kk][j], s, 0, 0, 0);
            }
        }
        return s;
    }
    __device__ __forceinline__ void values(char *tile, const f32x4 (&p)[NH], f32x4 (&o)[D / 16])
    {
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row = 16 * h + i * RW + lane / CR;
                *reinterpret_cast<f32x4 *>(tile + row * ROW + ((lane % CR) ^ swizzle(row)) * 16) = vx[h][i];
            }
        if constexpr (BF) {
            StepRows<true, ST, D>::template product32<D, true>(tile, p[0], p[1], o, l16, lg);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 4 * lg + j;
                const uint32_t at = (uint32_t)(r * ROW + (((l16 >> 2) ^ swizzle(r)) * 16) + 4 * (l16 & 3));
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt)
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(*reinterpret_cast<const float *>(tile + (at ^ (uint32_t)(64 * dt))), p[0][j], o[dt], 0, 0, 0);
            }
        }
    }
};

// a row's result: 4 channels from c on
template <typename ST>
__device__ __forceinline__ void put(const DecodeParams &a, long row, int c, const f32x4 &o, float m, float l)
{
    const float inv = l == 0.f ? 0.f : 1.f / l;
    ST *const to = (ST *)a.out + row * a.D + c;
    if constexpr (sizeof(ST) == 2) {
        *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    } else {
        *reinterpret_cast<float4 *>(to) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    }
    if (c == 0) {
        const float z = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);  // (base 2)
        if (a.lse) a.lse[row] = z * kLn2;
        a.lse2[row] = z;
    }
}

// Waves to a SIMD that the registers are shared out for, and so workgroups of the first launch: all that are on the CUs together.  What the waves of
// a CU have on their way decides (4 bits, 128 channels: 8.7 KB a wave in 168 registers).
constexpr int occupancy(bool four, int bytes, int D) { return D == 64 ? (four && bytes == 4 ? 3 : 4) : four && bytes == 2 ? 3 : 2; }

// SOLO: a workgroup a tile and no second launch, for caches that are a few steps long
template <bool FOUR, typename ST, int D, bool LISTED, bool TALLY, bool SOLO>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(occupancy(FOUR, sizeof(ST), D), occupancy(FOUR, sizeof(ST), D)))) void
decode_attend_kernel(const DecodeParams a)
{
    using R = StepRows<FOUR, ST, D>;
    constexpr int NH = R::NH, STEP = 16 * NH, C4 = D / 4;  // a step: a unit
    __shared__ __attribute__((aligned(1024))) char tiles[kWaves][64 * D];
    __shared__ float ml[kWaves][kQ][2];
    __shared__ int start[SOLO ? 1 : kMaxB + 1];
    __shared__ int wave_tot[kWaves];
    __shared__ float lse2[SOLO && TALLY ? kQ : 1];
    const int wave = scalar(threadIdx.x / kWave), me = blockIdx.x * kWaves + wave;
    LinePlan plan;
    LineTile w;
    int u0, n_steps;
    LineShares sh;
    if constexpr (SOLO) {
        const int HR = a.H * a.RT, hr = blockIdx.x % HR;
        w.b = blockIdx.x / HR, w.h = hr / a.RT, w.rt = hr % a.RT;
        w.L = scalar(length_of(a, w.b));
        w.s0 = 0, w.s1 = units_of(a, w.L);
        u0 = wave * w.s1 / kWaves, n_steps = (wave + 1) * w.s1 / kWaves - u0;
    } else {
        plan.make(a, start, wave_tot);
        sh = LineShares(plan.sum, a.H * a.RT, a.groups, a.three);
        if (blockIdx.x == 0) {  // for the second launch
            for (int b = threadIdx.x; b < a.B; b += kThreads) a.start[b] = plan.begin(b);
            if (threadIdx.x == 0) a.start[a.B] = plan.sum;
        }
        if (me >= sh.n) return;  // (a workgroup with such a wave has no results put together)
        u0 = sh.begin(me), n_steps = sh.begin(me + 1) - u0;
        w = plan.find(a, u0);
    }
    R r;
    r.lane = lane_id(), r.l16 = r.lane & 15, r.lg = r.lane >> 4;
    char *const tile = tiles[wave];
    const float cs = a.scale * kLog2e;

    auto base_of = [&](const LineTile &w) { return (long)(w.b * a.Hkv + w.h / (a.H / a.Hkv)) * a.Tcap; };
    auto query_of = [&](const LineTile &w) { return (long)w.b * a.Hq + w.h * a.G + w.rt * kQ; };  // the first one's row
    auto rows_of = [&](const LineTile &w) { return min(a.G - w.rt * kQ, kQ); };
    auto token_of = [&](const LineTile &w, int i) { return (u0 + i - w.s0) * STEP; };
    auto look_up = [&](const LineTile &w, int i) -> StepWhere<NH> {  // (past the last step: no rows)
        StepWhere<NH> x;
        const int t = token_of(w, i);
        const int32_t *list = LISTED ? a.idx + (long)(w.b * a.H + w.h) * a.K : nullptr;
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            int row = t + 16 * h;
            if constexpr (LISTED) {
                const int slot = row >> a.shift, page = i < n_steps && slot < a.K ? scalar(list[slot]) : -1;
                row = page < 0 || page >= (a.Tcap >> a.shift) ? a.Tcap : (page << a.shift) + (row & ((1 << a.shift) - 1));
            }
            const int left = w.L - row;
            x.valid[h] = scalar(i >= n_steps || left < 0 ? 0 : left < 16 ? left : 16);
            x.at[h] = scalar(x.valid[h] ? row : 0);
        }
        return x;
    };
    StepWhere<NH> x = look_up(w, 0);
    r.load_k(a, base_of(w), x);
    r.load_q((const ST *)a.q + (query_of(w) + (r.l16 < rows_of(w) ? r.l16 : 0)) * D, r.l16 < rows_of(w));
    r.load_v(a, base_of(w), x);
    // (now that the first rows are on their way) whether the workgroup's four shares are in one tile, so that their results are put together, and all of it
    bool together = true, whole = true;
    if constexpr (!SOLO) {
        const int g0 = sh.begin(blockIdx.x * kWaves), g1 = sh.begin((blockIdx.x + 1) * kWaves);
        together = (int)(blockIdx.x + 1) * kWaves <= sh.n && g0 >= w.s0 && g1 <= w.s1;
        whole = g0 == w.s0 && g1 == w.s1;
    }
    f32x4 o[D / 16];
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int i = 0; i < n_steps; ++i) {
        const int rows = rows_of(w);
        const long q_row = query_of(w);
        f32x4 s[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) s[h] = r.scores(h) * cs;
        const bool ends = i + 1 == n_steps || u0 + i + 1 >= w.s1;  // the tile, or the share
        LineTile then = w;
        if (!SOLO && ends && i + 1 < n_steps) {
            then = plan.find(a, u0 + i + 1);
            r.load_q((const ST *)a.q + (query_of(then) + (r.l16 < rows_of(then) ? r.l16 : 0)) * D, r.l16 < rows_of(then));
        }
        const StepWhere<NH> next = look_up(then, i + 1);
        r.load_k(a, base_of(then), next);
        float mx = -INFINITY;
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const int sees = x.valid[h] - 4 * r.lg;  // of the lane's four
            if (x.valid[h] < 16) {
#pragma unroll
                for (int j = 0; j < 4; ++j) s[h][j] = j < sees ? s[h][j] : -INFINITY;
            }
            if constexpr (TALLY) {
                if (r.l16 < rows) *reinterpret_cast<f32x4 *>(a.z + (q_row + r.l16) * a.z_row + token_of(w, i) + 16 * h + 4 * r.lg) = s[h];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, s[h][j]);
        }
        mx = quad_max(mx);
        if (__any(mx - m > kSlack)) {  // (-inf from -inf compares false)
            const float top = (mx - m > kSlack) ? mx : m, f = (m == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m - top);
            l *= f;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) o[dt] *= f;
            m = top;
        }
        const float bias = (m == -INFINITY) ? 0.f : m;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[h][j] = __builtin_amdgcn_exp2f(s[h][j] - bias);
                l += s[h][j];
            }
        r.values(tile, s, o);
        x = next;
        r.load_v(a, base_of(then), x);
        if (SOLO || !ends) continue;
        if (!together) {
            l = quad_sum(l);
            const int from = max(u0, w.s0), to = u0 + i + 1;
            const long slot = 2l * me + (from == w.s0 ? 1 : 0);  // a tile that began in another share: the first of two records
            if (r.l16 < rows) {
                if (from == w.s0 && to == w.s1) {
#pragma unroll
                    for (int dt = 0; dt < D / 16; ++dt) put<ST>(a, q_row + r.l16, 16 * dt + 4 * r.lg, o[dt], m, l);
                } else {
#pragma unroll
                    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4 *>(a.rec_o + (slot * a.rows + r.l16) * D + 16 * dt + 4 * r.lg) = o[dt];
                    if (r.lg == 0) *reinterpret_cast<float2 *>(a.rec_ml + (slot * a.rows + r.l16) * 2) = make_float2(m, l);
                }
            }
            if (i + 1 < n_steps) {
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
                m = -INFINITY, l = 0.f;
            }
        }
        w = then;
    }
    if (!together) return;
    l = quad_sum(l);
    if (r.lg == 0) ml[wave][r.l16][0] = m, ml[wave][r.l16][1] = l;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4 *>(tile + r.l16 * D * 4 + ((4 * dt + r.lg) ^ r.l16) * 16) = o[dt];
    __syncthreads();
    const long slot = 2l * kWaves * blockIdx.x;
    for (int e = threadIdx.x; e < rows_of(w) * C4; e += kThreads) {
        const int row = e / C4, c4 = e % C4;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) top = fmaxf(top, ml[i][row][0]);
        f32x4 out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const float mi = ml[i][row][0], li = ml[i][row][1];
            if (mi == -INFINITY && li == 0.f) continue;  // saw nothing
            const float f = mi == top ? 1.f : __builtin_amdgcn_exp2f(mi - top);
            sum += li * f;
            out += *reinterpret_cast<const f32x4 *>(tiles[i] + row * D * 4 + (c4 ^ row) * 16) * f;
        }
        if (whole) {
            put<ST>(a, query_of(w) + row, 4 * c4, out, top, sum);
        } else {
            *reinterpret_cast<f32x4 *>(a.rec_o + (slot * a.rows + row) * D + 4 * c4) = out;
            if (c4 == 0) *reinterpret_cast<float2 *>(a.rec_ml + (slot * a.rows + row) * 2) = make_float2(top, sum);
        }
        if (SOLO && TALLY && c4 == 0) lse2[row] = sum == 0.f ? 0.f : top + __builtin_amdgcn_logf(sum);  // (0: of scores that are all -inf)
    }
    if constexpr (SOLO && TALLY) {  // all of the KV head's queries are here (RT = 1)
        __syncthreads();
        const int rows = rows_of(w);
        float *const to = a.tally + (long)(w.b * a.Hkv + w.h) * a.Tcap;
        for (int t = 4 * threadIdx.x; t < w.L; t += 4 * kThreads) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int g = 0; g < rows; ++g) {
                const f32x4 z = *reinterpret_cast<const f32x4 *>(a.z + (query_of(w) + g) * a.z_row + t) - lse2[g];
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += __builtin_amdgcn_exp2f(z[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t + j < w.L) to[t + j] = (t + j >= w.L - a.fresh ? 0.f : to[t + j]) + sum[j];
        }
    }
}

// The records of the tile of units s0 .. s1 - 1, in their order: of single waves, of workgroups that are all inside it, of single waves.
struct TileRecords {
    int first, count, whole0, whole1;  // whole0 .. whole1 - 1: the workgroups inside

    __device__ __forceinline__ TileRecords(const LineShares &sh, int s0, int s1)
    {
        first = sh.of(s0);
        const int last = sh.of(s1 - 1);
        const int from = sh.begin(first) >= s0 ? first : first + 1, to = sh.begin(last + 1) <= s1 ? last + 1 : last;  // shares inside
        whole0 = (from + kWaves - 1) / kWaves, whole1 = to / kWaves;
        if (whole0 >= whole1) whole0 = whole1 = 1 << 28;  // none
        count = whole1 == 1 << 28 ? last - first + 1 : whole0 * kWaves - first + whole1 - whole0 + last + 1 - whole1 * kWaves;
    }
    __device__ __forceinline__ long slot(int i) const
    {
        const int singles = whole0 * kWaves - first;
        if (i >= singles && i < singles + whole1 - whole0) return 2l * kWaves * (whole0 + i - singles);
        const int share = i < singles ? first + i : whole1 * kWaves + i - (singles + whole1 - whole0);
        return 2l * share + (share == first ? 1 : 0);
    }
};

__device__ __forceinline__ void join(float &m, float &l, f32x4 &o, float m1, float l1, const f32x4 &o1)
{
    if (m1 == -INFINITY && l1 == 0.f) return;
    const float top = fmaxf(m, m1), f0 = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), f1 = m1 == top ? 1.f : __builtin_amdgcn_exp2f(m1 - top);
    m = top;
    l = l * f0 + l1 * f1;
    o = o * f0 + o1 * f1;
}

// Workgroups 0 .. B Hq - 1 join the records of a query each; the others, 1024 tokens of a KV head each, add its queries' weights to the tally.
template <typename ST, int D>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(const DecodeParams a)
{
    constexpr int C4 = D / 4, NG = kThreads / C4;
    __shared__ float part[NG][D], part_ml[NG][2];
    __shared__ float lse2[kThreads];
    const int HR = a.H * a.RT;
    const LineShares sh(a.start[a.B], HR, a.groups, a.three);
    const int rows = a.B * a.Hq;
    if ((int)blockIdx.x < rows) {
        const int row = blockIdx.x, b = row / a.Hq, hq = row - b * a.Hq, h = hq / a.G, g = hq - h * a.G, rt = g / kQ, r = g % kQ;
        const int n = a.start[b + 1] - a.start[b], s0 = a.start[b] * HR + (h * a.RT + rt) * n;
        const int c4 = threadIdx.x % C4, grp = threadIdx.x / C4;
        float m = -INFINITY, l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        if (n == 0) {
            if (grp == 0) put<ST>(a, row, 4 * c4, o, m, l);
            return;
        }
        const TileRecords rec(sh, s0, s0 + n);
        if (rec.count == 1) return;  // written as it is
        constexpr int AHEAD = 4;
        for (int i = grp; i < rec.count; i += AHEAD * NG) {
            float2 x[AHEAD];
            f32x4 v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                x[j] = make_float2(-INFINITY, 0.f);
                v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (i + j * NG < rec.count) {
                    const long at = rec.slot(i + j * NG) * a.rows + r;
                    x[j] = *reinterpret_cast<const float2 *>(a.rec_ml + at * 2);
                    v[j] = *reinterpret_cast<const f32x4 *>(a.rec_o + at * D + 4 * c4);
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) join(m, l, o, x[j].x, x[j].y, v[j]);
        }
        *reinterpret_cast<f32x4 *>(&part[grp][4 * c4]) = o;
        if (c4 == 0) part_ml[grp][0] = m, part_ml[grp][1] = l;
        __syncthreads();
        if (grp == 0) {
#pragma unroll
            for (int i = 1; i < NG; ++i) join(m, l, o, part_ml[i][0], part_ml[i][1], *reinterpret_cast<const f32x4 *>(&part[i][4 * c4]));
            put<ST>(a, row, 4 * c4, o, m, l);
        }
        return;
    }
    // ---- the tally ----
    const int slices = (a.Tcap + 4 * kThreads - 1) / (4 * kThreads), e = blockIdx.x - rows, bh = e / slices, b = bh / a.Hkv, h = bh - b * a.Hkv;
    const int t0 = (e - bh * slices) * 4 * kThreads, L = length_of(a, b);
    if (t0 >= L) return;
    const int n = a.start[b + 1] - a.start[b], lane = lane_id(), wave = threadIdx.x / kWave;
    const int t = t0 + 4 * threadIdx.x;
    float w[4] = {0.f, 0.f, 0.f, 0.f}, had[4];
    float *const to = a.tally + (long)bh * a.Tcap + t;
    // what does not depend on the log-sum-exps is on its way before they are worked out: the tally and the scores of the first queries
    constexpr int AHEAD = 4;
    float4 scores[AHEAD];
    const float *const z0 = a.z + ((long)b * a.Hq + h * a.G) * a.z_row + t;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) scores[i] = t < L && i < a.G ? *reinterpret_cast<const float4 *>(z0 + (long)i * a.z_row) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 4; ++j) had[j] = t + j < L - a.fresh ? to[j] : 0.f;
    auto add = [&](const float4 &x, float z) {
        const float s = z == -INFINITY ? 0.f : z;
        w[0] += __builtin_amdgcn_exp2f(x.x - s), w[1] += __builtin_amdgcn_exp2f(x.y - s);
        w[2] += __builtin_amdgcn_exp2f(x.z - s), w[3] += __builtin_amdgcn_exp2f(x.w - s);
    };
    for (int g0 = 0; g0 < a.G; g0 += kThreads) {  // (more than 256 queries to a KV head: by turns)
        const int n_g = min(a.G - g0, kThreads);
        for (int i = wave; i < n_g; i += kWaves) {
            const int g = g0 + i, rt = g / kQ, r = g % kQ;
            const int s0 = a.start[b] * HR + (h * a.RT + rt) * n;
            const TileRecords rec(sh, s0, s0 + n);
            float z;
            if (rec.count == 1) {
                z = a.lse2[(long)b * a.Hq + h * a.G + g];
            } else {
                float m = -INFINITY, l = 0.f;
                for (int x = lane; x < rec.count; x += kWave) {
                    const float2 y = *reinterpret_cast<const float2 *>(a.rec_ml + (rec.slot(x) * a.rows + r) * 2);
                    f32x4 none = {0.f, 0.f, 0.f, 0.f};
                    join(m, l, none, y.x, y.y, none);
                }
                const float top = wave_max(m);
                l = wave_sum(l * __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top)));
                z = l == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(l);
            }
            if (lane == 0) lse2[i] = z;
        }
        __syncthreads();
        if (t < L) {
            if (g0 == 0) {
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (i < n_g) add(scores[i], lse2[i]);
            }
#pragma unroll 4
            for (int i = g0 == 0 ? AHEAD : 0; i < n_g; ++i) add(*reinterpret_cast<const float4 *>(z0 + (long)(g0 + i) * a.z_row), lse2[i]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (t + j < L) to[j] = had[j] + w[j];
}

struct DecodeLayout {
    size_t ml, lse2, start, z, total;
    int z_row, groups, rows, unit;  // workgroups of the first launch; rows of a record
    bool three, solo;
};
// H, K: heads and pages of the lists; 0, 0: none
static DecodeLayout decode_layout(const rs_shape *s, bool four, int H, int K, bool tally)
{
    DecodeLayout x;
    const int heads = H ? H : s->Hkv, G = s->Hq / heads;
    x.rows = G < kQ ? G : kQ;
    x.unit = four ? 64 : s->dtype == RS_BF16 ? 32 : 16;
    const long tile = ((H ? (long)K * s->P : (long)s->Tcap) + x.unit - 1) / x.unit, tiles = (long)s->B * heads * ((G + kQ - 1) / kQ), units = tile * tiles;
    const long most = 256l * occupancy(four, (int)esize(s->dtype), s->D), need = (units + kWaves - 1) / kWaves;
    x.groups = (int)(need < most ? need : most);
    x.three = need >= most && most == 3 * 256;
    // A workgroup a tile, four of its units at a time, against even shares and a second launch (32 over 8 heads of 128 channels, tiles of 8 / 16 / 32 units, us):
    // 32 tiles, 4 bits 7.1 / 11.1 / 19.1 against 10.7 / 11.0 / 11.6, bfloat16 with tally 8.4 / 11.7 / 19.0 against 11.1 / 11.4 / 12.0; 512 tiles, 4 bits 11.7 / 18.0 / 30.0
    // against 20.7 / 25.7 / 36.9, bfloat16 with tally 15.6 / 26.3 / 54.9 against 20.6 / 32.7 / 58.6.  Longer tiles would gain too where all are alike, and lose much where they are not.
    x.solo = (tile <= 16 || (tile <= 32 && tiles >= 256)) && G <= kQ;  // (of a tile that is all of a KV head, the tally is its own too)
    const size_t records = (size_t)2 * x.groups * kWaves * x.rows;
    x.z_row = tally ? (s->Tcap + kUnit - 1) / kUnit * kUnit : 0;
    x.ml = RS_WS_CTRL_BYTES + align256(records * s->D * 4);
    x.lse2 = x.ml + align256(records * 8);
    x.start = x.lse2 + align256((size_t)s->B * s->Hq * 4);
    x.z = x.start + align256((size_t)(s->B + 1) * 4);
    x.total = x.z + (size_t)s->B * s->Hq * x.z_row * 4;
    return x;
}

// H, K: heads and pages of the lists; 0, 0: none
static int check_decode(const rs_shape *s, int H, int K)
{
    const bool listed = H != 0 || K != 0;
    const int st = check_rows(s, listed);
    if (st != RS_OK) return st;
    if (listed && ((H != s->Hq && H != s->Hkv) || K < 1 || K > s->Tcap / s->P)) return RS_INVALID_ARG;
    if (s->B > kMaxB || s->Tcap > (1 << 30)) return RS_UNSUPPORTED;
    const double heads = listed ? H : s->Hkv, tiles = heads * ((s->Hq / heads + kQ - 1) / kQ), tokens = listed ? (double)K * s->P : s->Tcap;
    // units of the line, and workgroups of the second launch (2^32 threads are more than a launch takes)
    if (s->B * tiles * (tokens / 16 + 1) > 2e9 || (double)s->B * s->Hq + (double)s->B * s->Hkv * (s->Tcap / 1024. + 1) >= 16777216.) return RS_UNSUPPORTED;
    return RS_OK;
}

template <bool FOUR, typename ST, int D, bool LISTED, bool TALLY>
static void decode_launch_form(const DecodeParams &a, bool solo, hipStream_t stream)
{
    if (solo) {
        decode_attend_kernel<FOUR, ST, D, LISTED, TALLY, true><<<(unsigned)(a.B * a.H * a.RT), kThreads, 0, stream>>>(a);
        return;
    }
    decode_attend_kernel<FOUR, ST, D, LISTED, TALLY, false><<<a.groups, kThreads, 0, stream>>>(a);
    const long slices = TALLY ? (long)a.B * a.Hkv * ((a.Tcap + 1023) / 1024) : 0;
    decode_join_kernel<ST, D><<<(unsigned)((long)a.B * a.Hq + slices), kThreads, 0, stream>>>(a);
}

template <bool FOUR, typename ST, int D>
static void decode_launch(const DecodeParams &a, bool solo, hipStream_t stream)
{
    if constexpr (FOUR) {
        if (a.idx) decode_launch_form<true, ST, D, true, false>(a, solo, stream);
        else if (a.tally) decode_launch_form<true, ST, D, false, true>(a, solo, stream);
        else decode_launch_form<true, ST, D, false, false>(a, solo, stream);
    } else {
        decode_launch_form<false, ST, D, false, true>(a, solo, stream);
    }
}

static int decode_run(const rs_shape *s, DecodeParams a, bool four, int H, int K, void *ws, hipStream_t stream)
{
    const DecodeLayout x = decode_layout(s, four, H, K, a.tally != nullptr);
    char *const w = (char *)ws;
    a.rec_o = (float *)(w + RS_WS_CTRL_BYTES), a.rec_ml = (float *)(w + x.ml), a.lse2 = (float *)(w + x.lse2);
    a.start = (int *)(w + x.start), a.z = (float *)(w + x.z), a.z_row = x.z_row;
    a.B = s->B, a.Hq = s->Hq, a.Hkv = s->Hkv, a.D = s->D, a.Tcap = s->Tcap;
    a.H = a.idx ? H : s->Hkv, a.G = s->Hq / a.H, a.RT = (a.G + kQ - 1) / kQ, a.K = K;
    a.shift = a.idx ? __builtin_ctz((unsigned)s->P) : 0;
    a.list_units = a.idx ? (int)(((long)K * s->P + x.unit - 1) / x.unit) : 0;
    a.groups = x.groups, a.three = x.three, a.rows = x.rows, a.unit = x.unit;
    const bool bf = s->dtype == RS_BF16;
    if (four) {
        if (bf && s->D == 128) decode_launch<true, bf16, 128>(a, x.solo, stream);
        else if (bf) decode_launch<true, bf16, 64>(a, x.solo, stream);
        else if (s->D == 128) decode_launch<true, float, 128>(a, x.solo, stream);
        else decode_launch<true, float, 64>(a, x.solo, stream);
    } else {
        if (bf && s->D == 128) decode_launch<false, bf16, 128>(a, x.solo, stream);
        else if (bf) decode_launch<false, bf16, 64>(a, x.solo, stream);
        else if (s->D == 128) decode_launch<false, float, 128>(a, x.solo, stream);
        else decode_launch<false, float, 64>(a, x.solo, stream);
    }
    return launch_status();
}

}  // namespace rs

using namespace rs;

extern "C" {

size_t kv4_attn_decode_workspace_bytes(const rs_shape *s, int32_t H_idx, int32_t K, int32_t with_tally)
{
    return check_decode(s, H_idx, K) == RS_OK ? decode_layout(s, true, H_idx, K, with_tally != 0).total : 0;
}

int32_t kv4_attn_decode(const rs_shape *s, const void *q, const uint8_t *k4, const uint8_t *k4_scale, const uint8_t *v4, const uint8_t *v4_scale,
                        const int32_t *len, float scale, const int32_t *idx, int32_t H_idx, int32_t K, float *tally, int32_t n_fresh, void *out,
                        float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    if (!idx) H_idx = K = 0;
    else if (H_idx < 1 || K < 1) return RS_INVALID_ARG;
    const int st = check_decode(s, H_idx, K);
    if (st != RS_OK) return st;
    if (!q || !k4 || !k4_scale || !v4 || !v4_scale || !len || !out || (idx && tally) || (tally && n_fresh < 0)) return RS_INVALID_ARG;
    for (const void *x : {q, (const void *)k4, (const void *)k4_scale, (const void *)v4, (const void *)v4_scale, (const void *)len, (const void *)idx,
                          (const void *)tally, (const void *)out, (const void *)lse_out})
        if (!aligned16(x)) return RS_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < decode_layout(s, true, H_idx, K, tally != nullptr).total) return RS_WORKSPACE_TOO_SMALL;
    DecodeParams a = {};
    a.q = q, a.k = k4, a.v = v4, a.ks = k4_scale, a.vs = v4_scale, a.len = len, a.idx = idx, a.out = out, a.lse = lse_out, a.tally = tally;
    a.fresh = n_fresh, a.scale = scale;
    return decode_run(s, a, true, H_idx, K, ws, (hipStream_t)stream);
}

size_t attn_decode_tally_workspace_bytes(const rs_shape *s) { return check_decode(s, 0, 0) == RS_OK ? decode_layout(s, false, 0, 0, true).total : 0; }

int32_t attn_decode_tally(const rs_shape *s, const void *q, const void *k_cache, const void *v_cache, const int32_t *len, float scale, float *tally,
                          int32_t n_fresh, void *out, float *lse_out, void *ws, size_t ws_bytes, void *stream)
{
    const int st = check_decode(s, 0, 0);
    if (st != RS_OK) return st;
    if (!q || !k_cache || !v_cache || !len || !tally || !out || n_fresh < 0) return RS_INVALID_ARG;
    for (const void *x : {q, k_cache, v_cache, (const void *)len, (const void *)tally, (const void *)out, (const void *)lse_out})
        if (!aligned16(x)) return RS_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < decode_layout(s, false, 0, 0, true).total) return RS_WORKSPACE_TOO_SMALL;
    DecodeParams a = {};
    a.q = q, a.k = k_cache, a.v = v_cache, a.len = len, a.out = out, a.lse = lse_out, a.tally = tally;
    a.fresh = n_fresh, a.scale = scale;
    return decode_run(s, a, false, 0, 0, ws, (hipStream_t)stream);
}

}  // extern "C"
