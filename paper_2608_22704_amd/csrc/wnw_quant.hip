// The 8-bit KV cache: quantising rows as they are written, reading them back, and attention over the
// bytes.  Layout and formats as in wnw.h.
//
//   quant_write_kernel   a tile of 64 rows of one head's K or V per work-group
//   quant_append_kernel  up to 16 new rows of one head's K or V per wavefront
//   quant_read_kernel    the same tiles back to fp32 / bf16
//   quant_token_kernel   attention of up to 32 query rows of a KV-head: every byte of K and V comes from HBM once
//   quant_wide_kernel    attention of many query rows: tiles become fp16 in shared memory once for 128 (64) rows
//   quant_merge_kernel, quant_merge_rows_kernel   join the parts of a cache that work-groups shared
//
// Bytes become fp16 on the way to the matrix cores, exactly: integers up to 127 and e4m3 numbers both fit.
// A query row is scaled by a power of two (its largest magnitude to 2^14 .. 2^15) and is then exact in fp16 as well, but
// for elements 2^28 times smaller than the largest, so logits carry fp32 rounding alone.  A softmax weight times its
// block's V scale is rounded to the sum of two fp16 (2^-22): one would be off by up to 2^-11, and 7 % of bf16 outputs would
// then not be the fp32 ones rounded, which is what the flag promises (512 tokens would take 302 us instead of 377, 64 query
// rows 223 instead of 260, five tokens of d = 64 82 instead of 96, single tokens as long).  Sums, maxima and logits are fp32.
#include "wnw.h"
#include "wnw_internal.h"
#include "wnw_lds.h"

#include <math.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

namespace wnw {

namespace {

constexpr int QT = 64;          // rows of a tile
constexpr int Q_THREADS = 256;  // four wavefronts
constexpr float Q_LOG2E = 1.4426950408889634f;
constexpr float Q_LN2 = 0.6931471805599453f;
constexpr int Q_MAX_CAP = 1 << 24;
constexpr int64_t Q_MAX_GROUPS = 0xffffffffll / Q_THREADS;   // a launch has fewer than 2^32 threads

typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef float qf4_t __attribute__((ext_vector_type(4)));
typedef unsigned qu2_t __attribute__((ext_vector_type(2)));
typedef unsigned qu4_t __attribute__((ext_vector_type(4)));

// The cache and the layers of it that a call handles.
struct QuantGeo {
    int B, L, H, cap, l0, nl;
    int bsh;          // log2 of the rows per scale
    const uint8_t *k, *v;
    const float *ks, *vs;
    // head hd (of nl * H) of a call's layers in sequence b
    __host__ __device__ size_t head(int b, int hd) const { return ((size_t)b * L + l0) * H + hd; }
};

__device__ inline int q_clamp(int x, int hi)
{
    return min(max(x, 0), hi);
}

// ---- lanes -----------------------------------------------------------------------------------

__device__ inline unsigned uniform(unsigned v)
{
    return (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ inline float lane_f(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ inline unsigned lane_of(unsigned v, int lane)
{
    return (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}
// Inclusive scans over the wavefront's lanes by data-parallel moves: within rows of sixteen lanes, then across them.
template <typename F>
__device__ inline unsigned wave_scan_by(unsigned v, F f)
{
    v = f(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
    v = f(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
    v = f(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
    v = f(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
    v = f(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
    return f(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
}
__device__ inline unsigned wave_scan(unsigned v)
{
    return wave_scan_by(v, [](unsigned a, unsigned b) { return a + b; });
}
__device__ inline unsigned wave_sum(unsigned v)
{
    return (unsigned)__builtin_amdgcn_readlane((int)wave_scan(v), 63);
}
__device__ inline unsigned wave_max(unsigned v)
{
    return (unsigned)__builtin_amdgcn_readlane((int)wave_scan_by(v, [](unsigned a, unsigned b) { return max(a, b); }), 63);
}
// Over the wavefront's lanes, for every lane.
__device__ inline float wave_maxf(float v)
{
    auto step = [&](int u) { v = fmaxf(v, __int_as_float(u)); };
    step(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x111, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x112, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x114, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x118, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x142, 0xa, 0xf, false));
    step(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x143, 0xc, 0xf, false));
    return lane_f(v, 63);
}
__device__ inline float wave_sumf(float v)
{
    auto step = [&](int u) { v += __int_as_float(u); };
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x111, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x112, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x114, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x118, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
    return lane_f(v, 63);
}

// ---- numbers ---------------------------------------------------------------------------------

// Scale of a block whose largest magnitude has the (fp32) bits `amax`; NaN if that is not finite.
template <int FMT>
__device__ inline float quant_scale(unsigned amax)
{
    if (amax >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    if constexpr (FMT == WNW_QUANT_INT8) return fmaxf(__uint_as_float(amax) / 127.f, 0x1p-126f);
    // amax = 1.m * 2^(e - 127) <= 448 s = 1.75 * 2^8 s
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((unsigned)max(e, 1) << 23);
}

// Four values under scale s (inv = 1 / s) to four bytes: nearest, ties to even.
// int8: the rounded product with inv is off by one at most, next to a tie; x - n s is exact in fp32 (n s is a
// multiple of s's last bit, and so is x unless n = 0), so comparing it with s / 2 decides.
// e4m3: s is a power of two, so the product is exact.
template <int FMT>
__device__ inline unsigned quant4(float x0, float x1, float x2, float x3, float s, float inv)
{
    if constexpr (FMT == WNW_QUANT_INT8) {
        float x[4] = {x0, x1, x2, x3}, n[4], e[4];
        const float half = 0.5f * s;
        float worst = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            n[i] = rintf(x[i] * inv);
            e[i] = fmaf(-n[i], s, x[i]);
            worst = fmaxf(worst, fabsf(e[i]));
        }
        if (worst >= half) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool odd = (int)n[i] & 1;
                if (e[i] > half || (e[i] == half && odd)) n[i] += 1.f;
                if (e[i] < -half || (e[i] == -half && odd)) n[i] -= 1.f;
            }
        }
        unsigned r = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) r |= (unsigned)((int)n[i] + 128) << (8 * i);
        return r;
    } else {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * inv, x1 * inv, 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x2 * inv, x3 * inv, lo, true);
    }
}

// Byte i of u as a number, before the scale.
template <int FMT>
__device__ inline float byte_value(unsigned u, int i)
{
    if constexpr (FMT == WNW_QUANT_INT8) return (float)((int)((u >> (8 * i)) & 255) - 128);
    return __builtin_amdgcn_cvt_f32_fp8((int)(u >> (8 * i)), 0);
}

// Four bytes held under scale `was`, rounded again under the larger scale `now`.  int8: the fp32 product has three roundings of
// 2^-24 and is below 127, off by 2^-15 at most; next to a tie a double decides.  A quotient x was / now near a tie is 1/2 or more, so
// that now < 2^8 was; with p the weight of was's last bit, 2 x was and (2 k + 1) now are multiples of p, and now < 2^32 p:
// unless equal they differ by p or more, and the quotient from k + 1/2 by p / (2 now) > 2^-33.  x was is exact in double and the
// division off by 2^-47 at most.
template <int FMT>
__device__ inline unsigned requant4(unsigned u, float was, float now, float ratio)
{
    if constexpr (FMT == WNW_QUANT_E4M3) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(byte_value<FMT>(u, 0) * ratio, byte_value<FMT>(u, 1) * ratio, 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(byte_value<FMT>(u, 2) * ratio, byte_value<FMT>(u, 3) * ratio, lo, true);
    } else {
        unsigned r = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = byte_value<FMT>(u, i), q = x * ratio;
            float n = rintf(q);
            if (fabsf(fabsf(q - n) - 0.5f) < 0x1p-14f) n = (float)rint((double)x * (double)was / (double)now);
            r |= (unsigned)((int)n + 128) << (8 * i);
        }
        return r;
    }
}

// Four bytes to four fp16, exactly.  int8: 0x64 in front of a byte u is the fp16 number 1024 + u.
template <int FMT>
__device__ inline void bytes_to_half(unsigned u, h2_t &lo, h2_t &hi)
{
    if constexpr (FMT == WNW_QUANT_INT8) {
        const h2_t bias = {(_Float16)1152, (_Float16)1152};
        lo = __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias;
        hi = __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias;
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.f, true);
    }
}
template <int FMT>
__device__ inline h8_t bytes_to_h8(unsigned a, unsigned b)
{
    h2_t p0, p1, p2, p3;
    bytes_to_half<FMT>(a, p0, p1);
    bytes_to_half<FMT>(b, p2, p3);
    return h8_t{p0.x, p0.y, p1.x, p1.y, p2.x, p2.y, p3.x, p3.y};
}

__device__ inline uint16_t to_bf16(float f)
{
    return __builtin_bit_cast(uint16_t, (__bf16)f);   // nearest, ties to even
}

// ---- writing ---------------------------------------------------------------------------------

// Work-group: one tile of 64 rows of one head, K (even) or V (odd).  Wavefront w has rows 16 w .. + 16; its lane has rows
// 4 rg .. + 4 (rg = 4 w + lane / 16) at dimensions E (lane % 16) .. + E, so that a block's maximum is one of a wavefront or of
// neighbours, and four of a lane's values are a dword of K or of V.
// Bound by memory: two bytes of a value come, one goes.  15512 rows of 240 KV-heads (2.86 GB) 492 us, 5.8 TB/s; 7756 of 72
// (429 MB) 90 us, 4.8 TB/s.  Stores past the caches made no difference.
// Dwords of four rows at one dimension, transposed through shared memory for whole tiles of V.
template <int DH>
struct QuantTileSmem {
    static constexpr int E = DH / 16;
    static constexpr int ROW = E * 16 + 4;   // dwords of a lane's E dimensions, padded: 4-way conflicts, not 16
    alignas(16) unsigned t[16 * ROW];
    // dword of rows 4 rg .. + 4 at dimension dg * E + j
    static __device__ int at(int dg, int j, int rg) { return dg * ROW + j * 16 + (rg & 3) * 4 + (rg >> 2); }
    // the 16 places from 16 h on of dimension d
    static __device__ int unit(int d, int h) { return d / E * ROW + d % E * 16 + h * 4; }
};

// E bf16 that are read once.
template <int E>
__device__ inline void load_row(uint16_t (&u)[E], const uint16_t *p)
{
    if constexpr (E == 8) {
        const qu4_t v = __builtin_nontemporal_load((const qu4_t *)p);
        __builtin_memcpy(u, &v, sizeof(u));
    } else {
        const qu2_t v = __builtin_nontemporal_load((const qu2_t *)p);
        __builtin_memcpy(u, &v, sizeof(u));
    }
}

template <int DH, int FMT>
__global__ __launch_bounds__(Q_THREADS) void quant_write_kernel(QuantGeo g, int n, int tiles, const uint16_t *__restrict__ kn,
                                                               const uint16_t *__restrict__ vn,
                                                               const int32_t *__restrict__ pos_dev,
                                                               const int32_t *__restrict__ count_dev)
{
    constexpr int E = DH / 16;
    __shared__ QuantTileSmem<DH> sm;
    __shared__ unsigned wmax[4];
    const bool is_v = blockIdx.x & 1;
    const int item = blockIdx.x >> 1, hd = item / tiles, b = hd / (g.nl * g.H);
    const int pos = q_clamp(pos_dev[b], g.cap), cnt = count_dev ? q_clamp(count_dev[b], n) : n, end = min(pos + cnt, g.cap);
    const int tile = pos / QT + (item - hd * tiles), row0 = tile * QT;
    if (pos >= end || row0 >= end) return;      // (no rows: the scale of pos's block may be another call's to write)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, dg = lane & 15, rg = tid >> 4;
    const size_t head = g.head(b, hd - b * g.nl * g.H);
    uint8_t *codes = const_cast<uint8_t *>(is_v ? g.v : g.k) + (head * g.cap + row0) * DH;
    float *scales = const_cast<float *>(is_v ? g.vs : g.ks) + ((head * g.cap) >> g.bsh);
    const uint16_t *src = (is_v ? vn : kn) + (size_t)hd * n * DH + (size_t)dg * E;

    const int gw = 1 << (g.bsh - 4);                     // wavefronts of a block
    const int first = row0 + wave / gw * gw * 16;        // the block's first row
    const bool has_old = first < pos, has_new = first < end && first + gw * 16 > pos;
    const bool whole = pos <= row0 && end >= row0 + QT;  // the tile has new rows only (uniform)
    const float was = has_old ? scales[first >> g.bsh] : 0.f;
    bool put[4], old[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + rg * 4 + i;
        put[i] = row >= pos && row < end;
        old[i] = has_new && row < pos;
    }
    float x[4][E];
    unsigned amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (put[i]) {
            uint16_t u[E];
            load_row<E>(u, src + (size_t)(row0 + rg * 4 + i - pos) * DH);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[i][e] = __uint_as_float((unsigned)u[e] << 16);
                amax = max(amax, __float_as_uint(x[i][e]) & 0x7fffffffu);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = 0.f;
        }
    }
    // The lane's bytes of earlier rows, in case they are to be rounded again: K's four rows, or V's dwords of four rows (of
    // one scale block), which are also what a dword with some new rows keeps.
    unsigned had[E] = {};
    const bool some_old = has_new && row0 + rg * 4 < pos, some_new = put[0] || put[1] || put[2] || put[3],
               all_new = put[0] && put[1] && put[2] && put[3];
    if (!whole) {
        if (!is_v) {
            if (some_old) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    __builtin_memcpy(&had[i * (E / 4)], __builtin_assume_aligned(codes + (size_t)(rg * 4 + i) * DH + dg * E, E), E);
            }
        } else if (some_old || (some_new && !all_new)) {
#pragma unroll
            for (int e = 0; e < E; ++e) had[e] = *((const unsigned *)(codes + (size_t)(dg * E + e) * QT) + (rg & 3) * 4 + (rg >> 2));
        }
    }
    amax = wave_max(amax);
    if (lane == 0) wmax[wave] = amax;
    __syncthreads();
    for (int w = wave / gw * gw; w < wave / gw * gw + gw; ++w) amax = max(amax, wmax[w]);
    float s = quant_scale<FMT>(amax);
    // a NaN on either side stays one
    if (has_old) s = was != was || s != s ? __uint_as_float(0x7fc00000u) : fmaxf(was, s);
    const bool good = s == s, grew = has_old && good && s > was;
    if (has_new && lane == 0 && wave % gw == 0) scales[first >> g.bsh] = s;
    const float inv = 1.f / s, ratio = was * inv;

    constexpr unsigned ZERO = FMT == WNW_QUANT_INT8 ? 0x80808080u : 0u;
    if (!is_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned w[E / 4];
            if (put[i]) {
#pragma unroll
                for (int e = 0; e < E; e += 4)
                    w[e / 4] = good ? quant4<FMT>(x[i][e], x[i][e + 1], x[i][e + 2], x[i][e + 3], s, inv) : ZERO;
            } else if (old[i] && grew) {
#pragma unroll
                for (int e = 0; e < E / 4; ++e) w[e] = requant4<FMT>(had[i * (E / 4) + e], was, s, ratio);
            }
            if (put[i] || (old[i] && grew))
                __builtin_memcpy(__builtin_assume_aligned(codes + (size_t)(rg * 4 + i) * DH + dg * E, E), w, E);
        }
        return;
    }
    if (whole) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            sm.t[sm.at(dg, e, rg)] = good ? quant4<FMT>(x[0][e], x[1][e], x[2][e], x[3][e], s, inv) : ZERO;
        __syncthreads();
#pragma unroll
        for (int u = tid; u < DH * 4; u += Q_THREADS)
            *(qu4_t *)(codes + (size_t)u * 16) = *(const qu4_t *)&sm.t[sm.unit(u >> 2, u & 3)];
        return;
    }
    // the dword's bytes: new, rounded again, or as they were
    unsigned mask_put = 0, mask_old = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mask_put |= put[i] ? 255u << (8 * i) : 0u;
        mask_old |= old[i] && grew ? 255u << (8 * i) : 0u;
    }
    if (!(mask_put | mask_old)) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        unsigned w = had[e];
        if (mask_old) w = (w & ~mask_old) | (requant4<FMT>(w, was, s, ratio) & mask_old);
        if (mask_put) w = (w & ~mask_put) | ((good ? quant4<FMT>(x[0][e], x[1][e], x[2][e], x[3][e], s, inv) : ZERO) & mask_put);
        *((unsigned *)(codes + (size_t)(dg * E + e) * QT) + (rg & 3) * 4 + (rg >> 2)) = w;
    }
}

// A few rows: n <= APPEND_ROWS, which lie in two groups of 16 rows (that start at multiples of 16) and two scale blocks at most.
// A wavefront has a head's K or V: what a launch of a work-group a tile spends its time on is starting wavefronts (the
// chip starts one in about 0.5 ns), of which three or four of four had nothing to write.  Lanes as there, for each of the
// groups; V's dwords of old and new rows take the new ones as bytes.  Old rows are only read when their scale grows.
// 7 rows of 720 KV-heads 12-19 -> 6-8 us, one row of 3840 22-36 -> 15 us, of 240 4-5 either way, of 8 (int8) 3.9.  Small
// calls wait for the chain position, rows, maximum, bytes; large ones for V's lines, of which a row has a byte each.
constexpr int APPEND_ROWS = 16;
template <int DH, int FMT>
__global__ __launch_bounds__(Q_THREADS) void quant_append_kernel(QuantGeo g, int n, int items, const uint16_t *__restrict__ kn,
                                                                const uint16_t *__restrict__ vn,
                                                                const int32_t *__restrict__ pos_dev,
                                                                const int32_t *__restrict__ count_dev)
{
    constexpr int E = DH / 16;
    constexpr unsigned ZERO = FMT == WNW_QUANT_INT8 ? 0x80808080u : 0u;
    const int item = (int)uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (item >= items) return;
    const bool is_v = item & 1;
    const int hd = item >> 1, b = hd / (g.nl * g.H);
    const int pos = q_clamp(pos_dev[b], g.cap), cnt = count_dev ? q_clamp(count_dev[b], n) : n, end = min(pos + cnt, g.cap);
    if (pos >= end) return;
    const int lane = threadIdx.x & 63, dg = lane & 15, r4 = lane >> 4;
    const size_t head = g.head(b, hd - b * g.nl * g.H);
    uint8_t *codes = const_cast<uint8_t *>(is_v ? g.v : g.k) + head * g.cap * DH;
    float *scales = const_cast<float *>(is_v ? g.vs : g.ks) + ((head * g.cap) >> g.bsh);
    const uint16_t *src = (is_v ? vn : kn) + (size_t)hd * n * DH + (size_t)dg * E;

    const int grp = pos >> 4, groups = end > (grp + 1) * 16 ? 2 : 1, block = pos >> g.bsh;
    const bool has_old = (block << g.bsh) < pos, two = (end - 1) >> g.bsh != block;   // two blocks: the groups' own
    const float was = has_old ? scales[block] : 0.f;
    auto row_of = [&](int u, int i) { return (grp + u) * 16 + r4 * 4 + i; };
    auto put = [&](int u, int i) { return row_of(u, i) >= pos && row_of(u, i) < end; };
    // dword of the lane's four rows of a group at its dimension e, and bytes of its row i
    auto at_v = [&](int group, int e) { return (size_t)(group >> 2) * QT * DH + (dg * E + e) * QT + r4 * 16 + (group & 3) * 4; };
    auto at_k = [&](int group, int i) { return (size_t)(group * 16 + r4 * 4 + i) * DH + dg * E; };

    uint16_t in[2][4][E];
    unsigned amax[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (u < groups) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < E; ++e) in[u][i][e] = 0;
                if (put(u, i)) load_row<E>(in[u][i], src + (size_t)(row_of(u, i) - pos) * DH);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (u < groups) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) amax[u] = max(amax[u], (unsigned)in[u][i][e] & 0x7fffu);
            amax[u] = wave_max(amax[u]) << 16;
        }
    }
    if (!two) amax[0] = amax[1] = max(amax[0], amax[1]);
    float s[2] = {quant_scale<FMT>(amax[0]), quant_scale<FMT>(amax[1])};
    // a NaN on either side stays one
    if (has_old) s[0] = was != was || s[0] != s[0] ? __uint_as_float(0x7fc00000u) : fmaxf(was, s[0]);
    if (!two) s[1] = s[0];
    if (lane == 0) {
        scales[block] = s[0];
        if (two) scales[block + 1] = s[1];
    }
    if (has_old && s[0] > was) {      // (false for a NaN)
        const float ratio = was * (1.f / s[0]);
        const int first = block << (g.bsh - 4);
        unsigned had[4][E];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int group = first + w, row = group * 16 + r4 * 4;
            if (row >= pos) continue;
            if (is_v) {
#pragma unroll
                for (int e = 0; e < E; ++e) had[w][e] = *(const unsigned *)(codes + at_v(group, e));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    __builtin_memcpy(&had[w][i * (E / 4)], __builtin_assume_aligned(codes + at_k(group, i), E), E);
            }
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int group = first + w, row = group * 16 + r4 * 4, old = pos - row;
            if (old <= 0) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                unsigned x = requant4<FMT>(had[w][e], was, s[0], ratio);
                if (is_v) {
                    const unsigned keep = old >= 4 ? 0u : ~0u << (8 * old);
                    *(unsigned *)(codes + at_v(group, e)) = (had[w][e] & keep) | (x & ~keep);
                } else if (e / (E / 4) < old)
                    *(unsigned *)(codes + at_k(group, e / (E / 4)) + e % (E / 4) * 4) = x;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (u >= groups) break;
        const float inv = 1.f / s[u];
        const bool good = s[u] == s[u];
        auto x = [&](int i, int e) { return __uint_as_float((unsigned)in[u][i][e] << 16); };
        if (is_v) {
            if (!(put(u, 0) || put(u, 1) || put(u, 2) || put(u, 3))) continue;
            unsigned w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = good ? quant4<FMT>(x(0, e), x(1, e), x(2, e), x(3, e), s[u], inv) : ZERO;
            if (put(u, 0) && put(u, 3)) {
#pragma unroll
                for (int e = 0; e < E; ++e) *(unsigned *)(codes + at_v(grp + u, e)) = w[e];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (put(u, i)) {
#pragma unroll
                        for (int e = 0; e < E; ++e) codes[at_v(grp + u, e) + i] = (uint8_t)(w[e] >> (8 * i));
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!put(u, i)) continue;
                unsigned w[E / 4];
#pragma unroll
                for (int e = 0; e < E; e += 4)
                    w[e / 4] = good ? quant4<FMT>(x(i, e), x(i, e + 1), x(i, e + 2), x(i, e + 3), s[u], inv) : ZERO;
                __builtin_memcpy(__builtin_assume_aligned(codes + at_k(grp + u, i), E), w, E);
            }
        }
    }
}

// ---- reading back ----------------------------------------------------------------------------

// The second argument is the outputs' type: fp32 results, rounded to bf16 (nearest, ties to even) where it says so.
template <int E>
__device__ inline void store_row(void *out, bool bf16, size_t elem, const float (&x)[E])
{
    if (bf16) {
        uint16_t u[E];
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = to_bf16(x[e]);
        __builtin_memcpy(__builtin_assume_aligned((uint16_t *)out + elem, E * 2), u, E * 2);
    } else
        __builtin_memcpy(__builtin_assume_aligned((float *)out + elem, 16), x, E * 4);
}

// Work-group and rows of a lane as in quant_write_kernel; its dimensions are E neighbours for bf16 and runs of four,
// 64 apart, for fp32, so that every store of a wavefront fills whole lines.  Everything passes through once: streamed
// (7756 rows of 72 KV-heads as bf16 77 -> 62 us; with eight neighbours as fp32, halves of lines, 185 -> 231 us).
// Bound by memory: 15512 rows of 240 KV-heads as bf16 (2.86 GB) 494 us, 5.8 TB/s; four sequences of up to 7756 rows of 72
// KV-heads as fp32 159 us; 64 rows of 720 KV-heads 13.5 us, of which starting 11520 wavefronts is 5.
template <int DH, int FMT, bool BF16>
__global__ __launch_bounds__(Q_THREADS) void quant_read_kernel(QuantGeo g, int n, int tiles, void *__restrict__ ko,
                                                              void *__restrict__ vo, const int32_t *__restrict__ pos_dev,
                                                              const int32_t *__restrict__ count_dev)
{
    constexpr int E = DH / 16, RUN = BF16 ? E : 4, RUNS = E / RUN;
    __shared__ QuantTileSmem<DH> sm;
    const bool both = ko && vo, is_v = both ? blockIdx.x & 1 : vo != nullptr;
    const int item = both ? blockIdx.x >> 1 : blockIdx.x, hd = item / tiles, b = hd / (g.nl * g.H);
    const int pos = q_clamp(pos_dev[b], g.cap), cnt = count_dev ? q_clamp(count_dev[b], n) : n, end = min(pos + cnt, g.cap);
    const int tile = pos / QT + (item - hd * tiles), row0 = tile * QT;
    if (row0 >= end) return;
    const int tid = threadIdx.x, wave = tid >> 6, d0 = (tid & 15) * RUN, rg = tid >> 4;
    const size_t head = g.head(b, hd - b * g.nl * g.H);
    const uint8_t *codes = (is_v ? g.v : g.k) + (head * g.cap + row0) * DH;
    const float s = (is_v ? g.vs : g.ks)[(head * g.cap + row0 + wave * 16) >> g.bsh];
    void *out = is_v ? vo : ko;
    const size_t to = (size_t)hd * n * DH + d0;
    auto dim = [&](int e) { return d0 + e / RUN * 64 + e % RUN; };
    unsigned w[4][E / 4];    // K: of the lane's four rows
    unsigned t[E];           // V: of the lane's dimensions, a byte for each of its rows
    if (!is_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row0 + rg * 4 + i < pos || row0 + rg * 4 + i >= end) continue;
#pragma unroll
            for (int j = 0; j < RUNS; ++j) {
                const uint8_t *p = codes + (size_t)(rg * 4 + i) * DH + d0 + j * 64;
                if constexpr (RUN == 8) {
                    const qu2_t u = __builtin_nontemporal_load((const qu2_t *)p);
                    w[i][0] = u.x;
                    w[i][1] = u.y;
                } else
                    w[i][j] = __builtin_nontemporal_load((const unsigned *)p);
            }
        }
    } else {
#pragma unroll
        for (int u = tid; u < DH * 4; u += Q_THREADS)
            *(qu4_t *)&sm.t[sm.unit(u >> 2, u & 3)] = __builtin_nontemporal_load((const qu4_t *)(codes + (size_t)u * 16));
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = sm.t[sm.unit(dim(e), rg & 3) + (rg >> 2)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + rg * 4 + i;
        if (row < pos || row >= end) continue;
        const size_t at = to + (size_t)(row - pos) * DH;
#pragma unroll
        for (int j = 0; j < RUNS; ++j) {
            float x[RUN];
#pragma unroll
            for (int e = 0; e < RUN; ++e)
                x[e] = s * (is_v ? byte_value<FMT>(t[j * RUN + e], i) : byte_value<FMT>(w[i][(j * RUN + e) / 4], e & 3));
            if constexpr (BF16) {
                uint16_t u[RUN];
#pragma unroll
                for (int e = 0; e < RUN; ++e) u[e] = to_bf16(x[e]);
                if constexpr (RUN == 8) {
                    qu4_t v;
                    __builtin_memcpy(&v, u, sizeof(v));
                    __builtin_nontemporal_store(v, (qu4_t *)((uint16_t *)out + at));
                } else {
                    qu2_t v;
                    __builtin_memcpy(&v, u, sizeof(v));
                    __builtin_nontemporal_store(v, (qu2_t *)((uint16_t *)out + at));
                }
            } else
                __builtin_nontemporal_store(qf4_t{x[0], x[1], x[2], x[3]}, (qf4_t *)((float *)out + at + j * 64));
        }
    }
}

// ---- attention -------------------------------------------------------------------------------

struct QuantAttend {
    QuantGeo g;
    int G, n, R;               // q-heads per KV-head, tokens, rows G * n of a KV-head: row r is token r / G, q-head r % G
    int W, RB, rsh;            // work-groups that share the batch's tiles, rows of a block and their log2
    int bf16;                  // outputs are bf16: the fp32 results, rounded as they are stored
    int nrb;                   // > 0: a work-group per block of rows, nrb blocks a head, nothing to join
    float inv_w;               // 1 / W
    const uint16_t *q;
    const int32_t *len, *count;
    void *out;
    float *lse, *mass;
    float *ws_o;               // [W][2][RB][d]: sums of weights times values of a block of rows over a piece of its cache
    float2 *ws_ml;             // [W][2][RB]: the piece's maximum (base 2) and sum of weights
    float2 *ws_row;            // masses: [rows] maximum and sum of rows whose cache is one piece
    float *ws_m;               // masses: [rows][cap / 64] the maximum that a tile's masses are relative to
    float scale;               // log2(e) / sqrt(d)
};

// The kernel's arguments once more, as memory: what only its last part needs is loaded there, and does not take scalar
// registers from the start (fetching instructions is what a short call waits for, and spills are instructions).
__device__ inline const QuantAttend &late_args()
{
    auto *p = (const __attribute__((address_space(4))) QuantAttend *)__builtin_amdgcn_kernarg_segment_ptr();
    __asm__ volatile("" : "+s"(p));
    return *(const QuantAttend *)p;
}

// Work of a batch: every block of RB query rows of every head has its sequence's tiles (one at least, so that an
// empty sequence's outputs are written).  W work-groups share them, whatever the lengths are, in one of two ways:
//   pieces  a block's tiles are cut into pieces of at most `pp` tiles, a work-group each;
//   line    all tiles in a line, in the order sequence, head, block of rows, tile, are cut into W equal parts (pp = 0), so that a
//           work-group's part may end one block and begin another.
// The line is even, but a second block costs a work-group about PIECE_COST tiles' time again (its queries, first tiles and
// the join of its wavefronts).  A block that is not whole leaves its result in the workspace, in the work-group's slot 1
// (its first tiles) or 0 (later ones), and a second kernel joins those.  With nrb > 0 there is none of this: every block has its
// own work-group.
constexpr int MIN_PIECE = 4;    // tiles of a piece at least, one per wavefront
constexpr int PIECE_COST = 10;

// a / b for 0 <= a < 2^24 and b > 0
__device__ inline int div24(int a, int b)
{
    int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
    const int r = a - q * b;
    q += r >= b ? 1 : 0;
    return q - (r < 0 ? 1 : 0);
}
// At least x / y, given inv = 1 / y rounded, and the same in every kernel.
__device__ inline unsigned at_least(unsigned x, float inv)
{
    return (unsigned)__fmul_rn(__fmul_rn((float)x, inv), 1.000001f) + 1;
}

struct QuantSeq {
    int len, cnt, tiles, nrb;   // rows, tokens of this call, tiles and blocks of rows of a head (0: none)
};
__device__ inline QuantSeq quant_seq(const QuantAttend &a, int b)
{
    QuantSeq q = {0, 0, 1, 0};
    if (b < a.g.B) {
        q.len = q_clamp(a.len[b], a.g.cap);
        q.cnt = a.count ? q_clamp(a.count[b], a.n) : a.n;
        q.tiles = max(1, (q.len + QT - 1) / QT);
        q.nrb = (q.cnt * a.G + a.RB - 1) >> a.rsh;
    }
    return q;
}

// f(x of this lane, x of lane ^ 16), and the same with lane ^ 32.
template <typename F>
__device__ inline float across_quarters(float x, F f)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
    auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ inline float quarters_max(float x)
{
    return across_quarters(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float quarters_sum(float x)
{
    return across_quarters(x, [](float a, float b) { return a + b; });
}
// How a batch is shared; every wavefront finds out by itself (lane i has the sequences i, i + 64, ...).
struct QuantShare {
    int heads, lane;
    int pp;              // tiles of a piece, or 0: the line
    unsigned per;        // items per work-group (tiles of the line, or 1 piece)
    unsigned total;      // items
    QuantSeq mine;       // sequence `lane`

    __device__ QuantSeq seq(const QuantAttend &a, int b0) const { return b0 == 0 ? mine : quant_seq(a, b0 + lane); }
    // items of a block of rows
    __device__ unsigned span(const QuantSeq &q) const { return pp ? (unsigned)div24(q.tiles + pp - 1, pp) : (unsigned)q.tiles; }
    __device__ unsigned work(const QuantSeq &q) const { return span(q) * (unsigned)(q.nrb * heads); }

    __device__ void init(const QuantAttend &a, int lane_)
    {
        heads = a.g.nl * a.g.H, lane = lane_, pp = 0;
        unsigned t = 0, units = 0, most = 0;
        if (a.g.B == 1) {       // (all of it scalar, and no other instructions to fetch)
            mine = quant_seq(a, 0);
            t = work(mine), units = (unsigned)(mine.nrb * heads), most = mine.nrb ? (unsigned)mine.tiles : 0u;
        } else {
            mine = quant_seq(a, lane);
            for (int b0 = 0; b0 < a.g.B; b0 += 64) {
                const QuantSeq q = seq(a, b0);
                t += work(q);
                units += (unsigned)(q.nrb * heads);
                most = max(most, q.nrb ? (unsigned)q.tiles : 0u);
            }
            t = wave_sum(t), units = wave_sum(units), most = wave_max(most);
        }
        total = t;
        per = max(at_least(t, a.inv_w), (unsigned)MIN_PIECE);
        if (units < (unsigned)a.W) {
            // pieces of at most p tiles are at most t / p + units
            const unsigned p = min(max(at_least(t, __builtin_amdgcn_rcpf((float)(a.W - units))), (unsigned)MIN_PIECE), most);
            if (p && piece_len((int)most, (int)p) <= (int)per + PIECE_COST) {
                pp = (int)p;
                per = 1;
                if (a.g.B == 1)
                    total = uniform(work(mine));
                else {
                    t = 0;
                    for (int b0 = 0; b0 < a.g.B; b0 += 64) t += work(seq(a, b0));
                    total = wave_sum(t);
                }
            }
        }
        per = uniform(per), pp = (int)uniform(pp);
    }
    // The sequence that item f (< total) belongs to, and the first of its items.
    __device__ int find(const QuantAttend &a, unsigned f, unsigned &start, QuantSeq &sq) const
    {
        if (a.g.B == 1) {
            start = 0;
            sq = {(int)uniform(mine.len), (int)uniform(mine.cnt), (int)uniform(mine.tiles), (int)uniform(mine.nrb)};
            return 0;
        }
        unsigned base = 0;
        for (int b0 = 0;; b0 += 64) {
            const QuantSeq q = seq(a, b0);
            const unsigned v = work(q), inc = wave_scan(v);
            const unsigned long long hit = __ballot(base + inc > f);
            if (hit) {
                const int at = __builtin_ctzll(hit);
                start = base + lane_of(inc - v, at);
                sq = {(int)lane_of(q.len, at), (int)lane_of(q.cnt, at), (int)lane_of(q.tiles, at), (int)lane_of(q.nrb, at)};
                return b0 + at;
            }
            base += lane_of(inc, 63);
        }
    }
    // Items of the sequences 0 .. end - 1.
    __device__ unsigned before(const QuantAttend &a, int end) const
    {
        if (end == 0) return 0;
        unsigned t = 0;
        for (int b0 = 0; b0 < end; b0 += 64) t += b0 + lane < end ? work(seq(a, b0)) : 0u;
        return wave_sum(t);
    }
    // Tiles of the pieces of a block of `tiles` tiles, cut evenly into pieces of at most p.
    __device__ static int piece_len(int tiles, int p)
    {
        const int n = div24(tiles + p - 1, p);
        return div24(tiles + n - 1, n);
    }
};

struct QuantRow {
    int row_of;      // index into [B][nl][H_q][n] of row r
    int vis;         // cache rows it sees; -1: not a row of this call
};
__device__ inline QuantRow quant_row(const QuantAttend &a, int hd, int r, int len, int cnt)
{
    const int i = a.n == 1 ? 0 : r / a.G, j = r - i * a.G;
    QuantRow q;
    q.row_of = (hd * a.G + j) * a.n + i;      // hd = (b * nl + l) * H + h
    q.vis = r < a.R && i < cnt ? max(0, min(len, len - cnt + i + 1)) : -1;
    return q;
}

__device__ inline float pow2i(int e)   // 2^e, e in -126 .. 127 (clamped from below)
{
    return __uint_as_float((unsigned)(max(e, -126) + 127) << 23);
}

// x 2^e for any e: one instruction, exact but for results below 2^-126.  V scales reach down to 2^-126, so that the factor
// alone, 2^15 over a scale, can be more than fp32 holds.
__device__ inline float times_pow2(float x, int e)
{
    return __builtin_amdgcn_ldexpf(x, e);
}

// The least e with all of the scales below 2^e, or -126 (a NaN, whose weights are NaN, has no say).
template <int N>
__device__ inline int scale_exp(const float (&s)[N])
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, s[i]);
    return (int)(__float_as_uint(top) >> 23) - 126;
}

// 2^x by the hardware instruction alone: results below 2^-126 flush to zero, which no sum here shows (every row's
// holds a term of 2^0).
__device__ inline float exp2_hw(float x)
{
    return __builtin_amdgcn_exp2f(x);
}

// What a logit is taken relative to when its maximum is m: a row that has seen nothing keeps -inf out of differences.
__device__ inline float finite_or_zero(float m)
{
    return m == -INFINITY ? 0.f : m;
}

// Eight weights as matrix operands, each the sum of two fp16.  The first is rounded towards zero by one instruction
// whose result is also what the second is the rest of: with (_Float16) in both places the compiler rounded the product
// with the V scale straight to fp16 in one of them, and where the other's fp32 value was a tie the two differed by a whole step.
__device__ inline void weights_to_half(const float (&p)[8], h8_t &hi, h8_t &lo)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const h2_t h = __builtin_bit_cast(h2_t, __builtin_amdgcn_cvt_pkrtz(p[i], p[i + 1]));
        hi[i] = h.x;
        hi[i + 1] = h.y;
        lo[i] = (_Float16)(p[i] - (float)h.x);
        lo[i + 1] = (_Float16)(p[i + 1] - (float)h.y);
    }
}

// Few query rows.  A work-group has its part of the batch's tiles; within a block of RB = 16 MT rows each wavefront takes
// tiles of 64 cache rows in turn, and MT times
//   S^T (16 keys x 16 rows) = K Q^T, K bytes straight from registers: lane (key l % 16, quarter l / 16) has 16 bytes of a
//   row per load, two matrix products of 32 dimensions; which dimensions is the same for Q;
//   O^T (16 dimensions x 16 rows) += V^T P^T: result element i of S^T is key 4 (l / 16) + i, so that two blocks'
//   results are P^T's operand as they stand, and the tile's layout gives V^T's: 16 bytes of one dimension.
// A wavefront's tile goes from global to shared memory without registers, each lane's bytes to a place that it alone reads:
// K's of the next tile are under way from the end of the first products on, V's from the end of the second.  Registers are
// left for two blocks of 16 rows and two wavefronts on every SIMD.
// The wavefronts' results meet in shared memory at the end, in the tiles' place.
// Memory bounds long caches (two operations a byte and query row), and the bytes in flight decide, 64 KB a work-group: 15512
// rows of 240 KV-heads, four query rows each, 151 us, 6.3 TB/s (a loop of loads alone reads 6.9), the matrix cores 12 % busy,
// fetched bytes 1.006 of the cache's; 91024 rows 865 us, 6.45 TB/s; five tokens of three sequences (20 query rows) 171 us,
// 5.6 TB/s.  Short calls wait for instructions, each fetched once, and for the chain length, tile, products, softmax,
// products: 8 KV-heads of 1064 rows 13 us, of 512 rows 8.5.
// Slower: tiles through registers instead of shared memory; two groups of wavefronts on a tile (a draft 269 -> 342 us).
template <int DH, int MT, int NW>
struct QuantTokenSmem {
    union {
        alignas(16) qu4_t tile[NW][2][DH / 16 * 64];    // [wavefront][K, V]
        alignas(16) float o[NW][32][DH];                // in the wavefront's own tile: others may still be reading theirs
    };
    float m[NW][16 * MT], l[NW][16 * MT];
    float2 whole[16 * MT];                             // maximum and 1 / sum of a block that is not to be joined
    static_assert(sizeof(tile) == sizeof(o) && MT <= 2, "a wavefront's results fit its tile");
    // 16-byte unit u of a row of o, spread over the banks
    static __device__ int unit(int row, int u) { return (u ^ (row & (DH / 4 - 1) & 15)) * 4; }
};

// As load_to_lds, past the caches that a stream does not fit.
__device__ inline void stream_to_lds(const void *base, unsigned off, unsigned lds)
{
    __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base) : "m0", "memory");
}

// A wave-uniform scale by the scalar unit, whose loads do not count among those of the tiles.
__device__ inline float scalar_load(const float *p, int i)
{
    return ((const __attribute__((address_space(4))) float *)p)[i];
}

// A query row whose largest magnitude has the bf16 bits amax: the power of two that takes it to 2^14 .. 2^15, and what
// turns its products with bytes into base-2 logits, before K's scale (NaN for a row that is not finite).
__device__ inline int query_shift(unsigned amax)
{
    return min(141 - (int)(amax >> 7), 126);
}
__device__ inline float query_up(unsigned amax)
{
    return pow2i(query_shift(amax));
}
__device__ inline float query_scale(unsigned amax, float scale)
{
    return amax >= 0x7f80u ? __uint_as_float(0x7fc00000u) : scale * pow2i(-query_shift(amax));
}
__device__ inline h8_t query_half(qu4_t u, float up)
{
    h8_t f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = (_Float16)(__uint_as_float(u[e] << 16) * up);
        f[2 * e + 1] = (_Float16)(__uint_as_float(u[e] & 0xffff0000u) * up);
    }
    return f;
}

// Q^T of a block of rows as fp16: column (row) lane % 16, quarter q has dimensions 64 j + 16 q + 8 e .. + 8 in f[2 j + e].
// Returns what turns products with bytes into base-2 logits, before K's scale.
template <int NJ>
__device__ inline float load_queries(const uint16_t *row, bool live, int quarter, float scale, h8_t (&f)[2 * NJ])
{
    qu4_t u[2 * NJ];
    unsigned amax = 0;
#pragma unroll
    for (int j = 0; j < 2 * NJ; ++j) {
        u[j] = live ? *(const qu4_t *)(row + (j >> 1) * 64 + quarter * 16 + (j & 1) * 8) : qu4_t{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = max(amax, max(u[j][e] & 0x7fffu, (u[j][e] >> 16) & 0x7fffu));
    }
    amax = max(amax, (unsigned)__shfl_xor((int)amax, 16));
    amax = max(amax, (unsigned)__shfl_xor((int)amax, 32));
    const float up = query_up(amax);
#pragma unroll
    for (int j = 0; j < 2 * NJ; ++j) f[j] = query_half(u[j], up);
    return query_scale(amax, scale);
}

// The raw block sums of a row, each relative to its tile's maximum, to shares of the whole: times 2^(tile's maximum - m) inv.
__device__ inline void mass_shares(const QuantAttend &a, size_t row, int len, int blocks, int from, int step, float m, float inv)
{
    const float mz = finite_or_zero(m);
    const int live = (len + (1 << a.g.bsh) - 1) >> a.g.bsh, tsh = 6 - a.g.bsh;
    float *to = a.mass + row * blocks;
    const float *mt = a.ws_m + row * (a.g.cap / QT);
    for (int j = from; j < blocks; j += step) to[j] = j < live ? to[j] * (exp2f(mt[j >> tsh] - mz) * inv) : 0.f;
}

// Tiles ta .. tb - 1 of block rb of head (b, hd)'s rows; slot: where a piece's result goes (-1: the block is whole).
template <int DH, int FMT, int MT, bool NTL, int NW>
__device__ inline void quant_token_block(const QuantAttend &a, QuantTokenSmem<DH, MT, NW> &sm, const QuantSeq &sq, int b, int hd,
                                         int rb, int ta, int tb, int slot)
{
    constexpr int NJ = DH / 64, ND = DH / 16, RB = 16 * MT;
    const QuantGeo &g = a.g;
    const int len = sq.len, cnt = sq.cnt;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const size_t head = g.head(b, hd - b * g.nl * g.H);
    const uint8_t *kh = g.k + head * g.cap * DH, *vh = g.v + head * g.cap * DH;
    const float *ks = g.ks + ((head * g.cap) >> g.bsh), *vs = g.vs + ((head * g.cap) >> g.bsh);

    // cache rows that the block's last and first row see
    const int seen = min(len, max(0, len - cnt + min(cnt - 1, min(rb * RB + RB - 1, a.R - 1) / a.G) + 1));
    const int full = (int)uniform(len - cnt + rb * RB / a.G + 1);
    const int t_end = (int)uniform(min(tb, (seen + QT - 1) / QT));
    int t = ta + wave;

    const unsigned lds_k = __builtin_amdgcn_readfirstlane(lds_address(sm.tile[wave][0])),
                   lds_v = __builtin_amdgcn_readfirstlane(lds_address(sm.tile[wave][1]));
    const unsigned off_k = col * DH + quarter * 16, off_v = col * QT + quarter * 16;
    auto load = [&](const uint8_t *base, unsigned off, unsigned lds) {
        NTL ? stream_to_lds(base, off, lds) : load_to_lds(base, off, lds);
    };
    auto load_k = [&](int t) {
        const uint8_t *p = kh + (size_t)t * QT * DH;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int j = 0; j < NJ; ++j) load(p, off_k + kb * 16 * DH + j * 64, lds_k + (kb * NJ + j) * 1024);
    };
    auto load_v = [&](int t) {
        const uint8_t *p = vh + (size_t)t * QT * DH;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) load(p, off_v + dt * 16 * QT, lds_v + dt * 1024);
    };
    if (t < t_end) {
        load_k(t);
        load_v(t);
    }

    QuantRow qr[MT];
    h8_t qf[MT][2 * NJ];
    float crow[MT], m[MT], sum[MT];
    int vexp[MT];              // o is in units of 2^(vexp - 15); V scales of the rows that the lane's row has seen are below 2^vexp
    qf4_t o[MT][ND];
#pragma unroll
    for (int r = 0; r < MT; ++r) {
        qr[r] = quant_row(a, hd, rb * RB + r * 16 + col, len, cnt);
        crow[r] = load_queries<NJ>(a.q + (size_t)qr[r].row_of * DH, qr[r].vis >= 0, quarter, a.scale, qf[r]);
        m[r] = -INFINITY;
        sum[r] = 0.f;
        vexp[r] = -126;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[r][dt] = qf4_t{0.f, 0.f, 0.f, 0.f};
    }
    for (; t < t_end; t += NW) {
        const int key0 = t * QT + quarter * 4;
        const bool masked = t * QT + QT > full;   // some row does not see all of the tile
        const bool more = t + NW < t_end;
        float s[MT][4][4], ksc[4], vsc[4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            ksc[kb] = scalar_load(ks, (t * QT + kb * 16) >> g.bsh);
            vsc[kb] = scalar_load(vs, (t * QT + kb * 16) >> g.bsh);
        }
        lds_loads_wait<ND>();       // K is there, V's ND loads may be under way
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            qf4_t c[MT] = {};
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const qu4_t u = sm.tile[wave][0][(kb * NJ + j) * 64 + lane];
                const h8_t k0 = bytes_to_h8<FMT>(u.x, u.y), k1 = bytes_to_h8<FMT>(u.z, u.w);
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    c[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[r][2 * j], c[r], 0, 0, 0);
                    c[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[r][2 * j + 1], c[r], 0, 0, 0);
                }
            }
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][kb][i] = c[r][i];
        }
        __builtin_amdgcn_sched_barrier(0);
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the bytes have been read
        if (more) load_k(t + NW);
        __builtin_amdgcn_sched_barrier(0);

        const int tile_exp = (int)uniform((unsigned)scale_exp(vsc));
        h8_t ph[MT][2], pl[MT][2];
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            // logits are x[kb][.] f[kb]; where masks are needed they are made here, and f is 1
            float (&x)[4][4] = s[r], f[4], w[4];
            int ve = tile_exp;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) f[kb] = crow[r] * ksc[kb], w[kb] = vsc[kb];
            if (masked) {
                // only blocks that the row sees count: a later row's scale must not take bits from its weights
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) w[kb] = t * QT + kb * 16 < qr[r].vis ? w[kb] : 0.f;
                ve = scale_exp(w);
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[kb][i] = key0 + kb * 16 + i < qr[r].vis ? x[kb][i] * f[kb] : -INFINITY;
                    f[kb] = 1.f;
                }
            }
            float mt = m[r];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
                mt = fmaxf(mt, fmaxf(fmaxf(x[kb][0], x[kb][1]), fmaxf(x[kb][2], x[kb][3])) * f[kb]);
            mt = quarters_max(mt);
            ve = max(ve, vexp[r]);
            if (__any(ve > vexp[r] || mt > m[r])) {
                const float alpha = exp2_hw(m[r] - finite_or_zero(mt)), f = times_pow2(alpha, vexp[r] - ve);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) o[r][dt] *= f;
                sum[r] *= alpha;
                m[r] = mt;
                vexp[r] = ve;
            }
            const float mz = finite_or_zero(m[r]);
            float bs[4];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[kb][i] = exp2_hw(fmaf(x[kb][i], f[kb], -mz));
                bs[kb] = (x[kb][0] + x[kb][1]) + (x[kb][2] + x[kb][3]);
            }
            sum[r] += (bs[0] + bs[1]) + (bs[2] + bs[3]);
            if (a.mass) {
                // block sums relative to m; the merge makes them shares
                const int nb = QT >> g.bsh;
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) bs[kb] = quarters_sum(bs[kb]);
                if (quarter == 0 && qr[r].vis >= 0) {
                    float *to = a.mass + (size_t)qr[r].row_of * (g.cap >> g.bsh) + (size_t)t * nb;
                    if (nb == 1)
                        to[0] = (bs[0] + bs[1]) + (bs[2] + bs[3]);
                    else if (nb == 2) {
                        to[0] = bs[0] + bs[1];
                        to[1] = bs[2] + bs[3];
                    } else {
#pragma unroll
                        for (int kb = 0; kb < 4; ++kb) to[kb] = bs[kb];
                    }
                    a.ws_m[(size_t)qr[r].row_of * (g.cap / QT) + t] = m[r];
                }
            }
            // P^T, times the V scales; a masked weight is 0 whatever the scale is
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                w[kb] = times_pow2(w[kb], 15 - ve);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[kb][i] *= w[kb];
            }
            if (masked) {
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[kb][i] = key0 + kb * 16 + i < qr[r].vis ? x[kb][i] : 0.f;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float p[8] = {x[2 * c][0],     x[2 * c][1],     x[2 * c][2],     x[2 * c][3],
                                    x[2 * c + 1][0], x[2 * c + 1][1], x[2 * c + 1][2], x[2 * c + 1][3]};
                weights_to_half(p, ph[r][c], pl[r][c]);
            }
        }
        if (more)
            lds_loads_wait<4 * NJ>();     // V is there, the next K may be under way
        else
            lds_loads_wait<0>();
        unsigned live[4] = {~0u, ~0u, ~0u, ~0u};
        const bool tail = FMT == WNW_QUANT_E4M3 && t * QT + QT > len;
        if (tail) {
            // bytes of dead rows may be e4m3's NaN
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                const int n = len - (key0 + kb * 16);
                live[kb] = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
            }
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            qu4_t u = sm.tile[wave][1][dt * 64 + lane];
            if (tail) u &= qu4_t{live[0], live[1], live[2], live[3]};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const h8_t v = bytes_to_h8<FMT>(u[2 * c], u[2 * c + 1]);
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[r][c], o[r][dt], 0, 0, 0);
                    o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl[r][c], o[r][dt], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) load_v(t + NW);
        __builtin_amdgcn_sched_barrier(0);
    }

#pragma unroll
    for (int r = 0; r < MT; ++r) {
        sum[r] = quarters_sum(sum[r]);
        if (quarter == 0) {
            sm.m[wave][r * 16 + col] = m[r];
            sm.l[wave][r * 16 + col] = sum[r];
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            qf4_t y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = times_pow2(o[r][dt][i], vexp[r] - 15);
            *(qf4_t *)&sm.o[wave][r * 16 + col][sm.unit(r * 16 + col, dt * 4 + quarter)] = y;
        }
    }
    __syncthreads();
    const QuantAttend &z = late_args();
    for (int row = threadIdx.x >> 4; row < RB; row += NW * 4) {
        const int d0 = (threadIdx.x & 15) * (DH / 16);
        const QuantRow rr = quant_row(z, hd, rb * RB + row, len, cnt);
        if (rr.vis < 0) continue;
        float mm = -INFINITY, ll = 0.f, x[DH / 16];
#pragma unroll
        for (int w = 0; w < NW; ++w) mm = fmaxf(mm, sm.m[w][row]);
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) x[e] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float lw = sm.l[w][row], f = lw == 0.f ? 0.f : exp2f(sm.m[w][row] - finite_or_zero(mm));   // 0: saw nothing
            ll += f * lw;
#pragma unroll
            for (int e = 0; e < DH / 16; e += 4) {
                const qf4_t y = *(const qf4_t *)&sm.o[w][row][sm.unit(row, (d0 + e) / 4)];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e + k] += f * y[k];
            }
        }
        if (slot >= 0) {
            const size_t at = (size_t)(blockIdx.x * 2 + slot) * RB + row;
            __builtin_memcpy(__builtin_assume_aligned(z.ws_o + at * DH + d0, 16), x, sizeof(x));
            if (d0 == 0) z.ws_ml[at] = make_float2(mm, ll);
        } else {
            const float inv = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
            for (int e = 0; e < DH / 16; ++e) x[e] *= inv;
            store_row<DH / 16>(z.out, z.bf16, (size_t)rr.row_of * DH + d0, x);
            if (d0 == 0) {
                if (z.lse) z.lse[rr.row_of] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * Q_LN2;
                if (z.mass) {
                    if (z.nrb)
                        sm.whole[row] = make_float2(mm, inv);
                    else
                        z.ws_row[rr.row_of] = make_float2(mm, ll);
                }
            }
        }
    }
    if (z.mass && z.nrb) {
        // nobody joins this block: its tiles' sums become shares here (n = 1: row r is q-head r)
        __syncthreads();
        const int rows = min(RB, z.R - rb * RB), blocks = z.g.cap >> z.g.bsh;
        for (int row = wave; row < rows; row += NW) {
            const float2 mi = sm.whole[row];
            mass_shares(z, (size_t)hd * z.G + rb * RB + row, len, blocks, lane, 64, mi.x, mi.y);
        }
    }
}

// Work-groups of NW wavefronts that a compute unit holds: of d = 128 two of four by shared memory, of d = 64 with one block of
// rows three by registers.  Eight are for launches that leave a compute unit to each work-group: a round of tiles is one
// wavefront's instructions one after the other, which two on a SIMD overlap.
template <int DH, int MT>
constexpr int token_held()
{
    return DH == 64 && MT == 1 ? 3 : 2;
}

// Runs f(sequence, b, head, block of rows, first tile, end tile, slot) for the work-group's part of a batch.
template <typename F>
__device__ inline void quant_parts(const QuantAttend &a, F f)
{
    QuantShare sh;
    QuantSeq sq;
    int b = 0, hd, rb, ta = 0, tb;
    unsigned i = 0, i1 = 0, start = 0;
    auto item = [&]() {
        const unsigned off = i - start, span = uniform(sh.span(sq));
        const unsigned unit = span == 1 ? off : sh.pp ? (unsigned)div24((int)off, (int)span) : off / span, at = off - unit * span;
        ta = (int)at;
        tb = (int)min(span, at + (i1 - i));
        i += tb - ta;
        if (sh.pp) {
            const int len = QuantShare::piece_len(sq.tiles, sh.pp);
            ta = min(sq.tiles, (int)at * len);
            tb = min(sq.tiles, ta + len);
        }
        hd = sq.nrb == 1 ? (int)unit : (int)unit / sq.nrb;
        rb = (int)unit - hd * sq.nrb;
        hd = (int)uniform(hd + b * sh.heads), rb = (int)uniform(rb), ta = (int)uniform(ta), tb = (int)uniform(tb);
    };
    if (a.nrb > 0) {
        hd = a.nrb == 1 ? (int)blockIdx.x : (int)blockIdx.x / a.nrb;
        rb = (int)blockIdx.x - hd * a.nrb;
        if (a.g.B > 1) b = hd / (a.g.nl * a.g.H);
        sq = quant_seq(a, b);
        if (rb >= sq.nrb) return;
        tb = sq.tiles;
    } else {
        sh.init(a, threadIdx.x & 63);
        i = blockIdx.x * sh.per;
        if (i >= sh.total) return;
        i1 = min(i + sh.per, sh.total);
        b = sh.find(a, i, start, sq);
        item();
    }
    for (;;) {
        f(sq, b, hd, rb, ta, tb, ta > 0 ? 0 : tb < sq.tiles ? 1 : -1);
        if (i >= i1) return;
        if (i - start >= sh.work(sq)) b = sh.find(a, i, start, sq);
        item();
        __syncthreads();
    }
}

template <int DH, int FMT, int MT, bool NTL, int NW>
__global__ __launch_bounds__(64 * NW, (NW == 8 ? 2 : token_held<DH, MT>())) void quant_token_kernel(QuantAttend a)
{
    __shared__ QuantTokenSmem<DH, MT, NW> sm;
    quant_parts(a, [&](const QuantSeq &sq, int b, int hd, int rb, int ta, int tb, int slot) {
        quant_token_block<DH, FMT, MT, NTL, NW>(a, sm, sq, b, hd, rb, ta, tb, slot);
    });
}

// Many query rows.  A work-group has blocks of RB = 128 rows, 32 for each of its four wavefronts; all of them use the same
// tiles of 64 cache rows, which two buffers in shared memory hold as fp16, so that a byte is converted once per 128
// rows.  While a tile is in use the next one's bytes, loaded a round before, are converted and written, and those of the
// one after it are on their way to registers.
//   S^T (32 keys x 32 rows) = K Q^T and O^T (32 dimensions x 32 rows) += V^T P^T by 32 x 32 x 16 products (see wnw_lds.h for
//   operands): a lane has 16 keys of ONE row, elements 0 .. 7 in the tile's 16-row block 2 k and 8 .. 15 in 2 k + 1, so that S^T's
//   elements are P^T's operand as they stand.
// KS = 2, for 33 to 64 rows: two wavefronts share 32 rows, each with half of every tile's keys, and join at the end (with
// two of four wavefronts idle instead: 64 rows of 240 KV-heads over 15512 rows 367 -> 260 us).
// A row's maximum m is raised, and its output and sum scaled, only when a logit exceeds it by LAZY (base 2): weights
// are up to 2^LAZY then, which fp16 has room for (a weight of 1 stands at 2^7 instead of 2^15, so that weights end at 2^-31 of the
// largest V scale seen, where the kernel for few rows has 2^-39).
// Bound by the matrix cores and the vector unit taking turns within the card's power limit: a wavefront's tile is 48
// products (1536 cycles; weights are two operands) and about 340 vector instructions, which the two work-groups of a compute unit
// overlap; the matrix cores are 47 % busy.  512 tokens of four heads over 15512 rows of 16 KV-heads 377-387 us with a join of 12, 665-680
// TFLOP/s or 1000-1020 with the second product of every weight; 1024 tokens over 8000 rows of 32 KV-heads 710-727 us, 700 and 1050
// TFLOP/s (a large product of the library: 1149 in bf16, 1107 in fp16).  After a pause the card's clocks take some milliseconds of
// such work to settle, with calls up to a quarter longer.  Fetched bytes are eight times the cache's (every XCD reads all of
// it), from the last-level cache.  Not kept, measured with one product for each weight: conversions between the products
// instead of before them (1.5 % faster, d = 64 2 % slower), raised priority around the products (2 %).
constexpr int WIDE_ROWS = 128;   // 2^7: see QuantAttend::rsh
constexpr int LAZY = 8;

// Tiles in shared memory: a row of K has its dimensions, a row of V (a dimension) the tile's rows, 16-byte unit 2 c + half
// with rows 4 half .. + 4 and 8 + 4 half .. + 4 of 16-row block c.  Rows are 16 bytes longer than their content: the eight lanes of
// a cycle, on one unit of eight rows, meet distinct banks, and every access of a lane is its base and a constant
// (with the units permuted by an exclusive or instead, their addresses took a tenth of the vector instructions).
template <int DH>
struct QuantWideSmem {
    static constexpr unsigned K_ROW = DH * 2 + 16, V_ROW = QT * 2 + 16, K_BYTES = QT * K_ROW, BUF = K_BYTES + DH * V_ROW;
    alignas(256) unsigned char tile[2][BUF];   // K, then V
};
// In the tiles' place at the end, where two wavefronts share 32 rows: sums, maximum and sum of weights of the second.
template <int DH>
struct QuantWideJoin {
    qf4_t o[2][DH / 8][64];
    float2 ml[2][64];
};
__device__ inline h8_t lds_read(unsigned at)
{
    return __builtin_bit_cast(h8_t, *(const __attribute__((address_space(3))) qu4_t *)(size_t)at);
}
__device__ inline void lds_write(unsigned at, qu4_t x)
{
    *(__attribute__((address_space(3))) qu4_t *)(size_t)at = x;
}

template <int FMT>
__device__ inline qu4_t convert8(unsigned a, unsigned b)
{
    return __builtin_bit_cast(qu4_t, bytes_to_h8<FMT>(a, b));
}

template <int DH, int FMT, int KS>
__device__ inline void quant_wide_block(const QuantAttend &a, QuantWideSmem<DH> &sm, const QuantSeq &sq, int b, int hd, int rb,
                                        int ta, int tb, int slot)
{
    constexpr int NS = DH / 16, ND = DH / 32, RB = WIDE_ROWS / KS, NB = 2 / KS;    // NB: blocks of 32 keys of a wavefront
    const QuantGeo &g = a.g;
    const int len = sq.len, cnt = sq.cnt;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int rows32 = KS == 2 ? wave & 1 : wave, key32 = KS == 2 ? wave >> 1 : 0;    // the wavefront's rows, and its keys of a tile
    const size_t head = g.head(b, hd - b * g.nl * g.H);
    const uint8_t *kh = g.k + head * g.cap * DH, *vh = g.v + head * g.cap * DH;
    const float *ks = g.ks + ((head * g.cap) >> g.bsh), *vs = g.vs + ((head * g.cap) >> g.bsh);

    // cache rows that the block's last and first row see
    const int seen = min(len, max(0, len - cnt + min(cnt - 1, min(rb * RB + RB - 1, a.R - 1) / a.G) + 1));
    const int full = (int)uniform(max(0, len - cnt + rb * RB / a.G + 1));
    const int t_end = (int)uniform(min(tb, (seen + QT - 1) / QT));

    // bytes of a tile: the thread has 32 (16) dimensions of one key, and 32 places of one dimension of V
    constexpr int KL = DH / 64;
    const int key_t = tid >> 2, part_t = tid & 3, d_t = tid >> 1, half_t = tid & 1;
    const bool has_v = DH == 128 || tid < 2 * DH;
    qu4_t kr[KL], vr[2];
    auto load = [&](int t) {
        const uint8_t *pk = kh + (size_t)t * QT * DH, *pv = vh + (size_t)t * QT * DH;
#pragma unroll
        for (int j = 0; j < KL; ++j) kr[j] = *(const qu4_t *)(pk + (key_t * DH + (part_t * KL + j) * 16));
        if (has_v) {
            vr[0] = *(const qu4_t *)(pv + (d_t * QT + half_t * 16));
            vr[1] = *(const qu4_t *)(pv + (d_t * QT + half_t * 16 + 32));
        }
    };
    using SM = QuantWideSmem<DH>;
    const unsigned lds = uniform(lds_address(sm.tile[0]));
    const unsigned k_put = lds + key_t * SM::K_ROW + part_t * KL * 32,
                   v_put = lds + SM::K_BYTES + d_t * SM::V_ROW + half_t * 16;
    const unsigned k_get = lds + (col + key32 * 32) * SM::K_ROW + half * 16,
                   v_get = lds + SM::K_BYTES + col * SM::V_ROW + half * 16 + key32 * 64;
    auto store = [&](int t, unsigned buf) {
#pragma unroll
        for (int j = 0; j < KL; ++j) {
            lds_write(k_put + j * 32 + buf, convert8<FMT>(kr[j].x, kr[j].y));
            lds_write(k_put + j * 32 + 16 + buf, convert8<FMT>(kr[j].z, kr[j].w));
        }
        if (has_v) {
            if (FMT == WNW_QUANT_E4M3 && t * QT + QT > len) {
                // bytes of dead rows may be e4m3's NaN
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int n = len - (t * QT + 16 * c + 4 * (half_t + 2 * j));
                        vr[j][c] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                    }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) lds_write(v_put + c * 32 + buf, convert8<FMT>(vr[0][c], vr[1][c]));
        }
    };
    if (ta < t_end) load(ta);

    const QuantRow qr = quant_row(a, hd, rb * RB + rows32 * 32 + col, len, cnt);
    h8_t qf[NS];
    float crow;
    {
        qu4_t u[NS];
        unsigned amax = 0;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            u[s] = qr.vis >= 0 ? *(const qu4_t *)(a.q + (size_t)qr.row_of * DH + s * 16 + half * 8) : qu4_t{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) amax = max(amax, max(u[s][e] & 0x7fffu, (u[s][e] >> 16) & 0x7fffu));
        }
        amax = max(amax, (unsigned)__shfl_xor((int)amax, 32));
        crow = query_scale(amax, a.scale);
        const float up = query_up(amax);
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[s] = query_half(u[s], up);
    }
    float m = -INFINITY, sum = 0.f;
    f32x16_t o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    int vexp = -126;           // o is in units of 2^(vexp + LAZY - 15); V scales of the rows that the lane's row has seen are below 2^vexp
    if (ta < t_end) {
        store(ta, 0);
        if (ta + 1 < t_end) load(ta + 1);
    }
    __syncthreads();
    // one tile, from the buffer at `buf`; the next one goes to the other.  MASKED: some row may not see all of the tile.
    auto round = [&](int t, auto buf_c, auto masked_c) {
        const unsigned buf = buf_c, other = SM::BUF - buf;
        constexpr bool MASKED = decltype(masked_c)::value;
        const int row = t * QT + key32 * 32;      // of the cache, the wavefront's first
        float f[2 * NB], vsc[2 * NB];
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c) {
            f[c] = crow * scalar_load(ks, (row + c * 16) >> g.bsh);
            vsc[c] = scalar_load(vs, (row + c * 16) >> g.bsh);
        }
        f32x16_t x[NB];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kb][i] = 0.f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
                x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_read(k_get + s * 32 + kb * 32 * SM::K_ROW + buf), qf[s], x[kb], 0,
                                                               0, 0);
        // element i of x[kb] is of key 32 kb + 8 (i / 4) + i % 4 from here; `vis` is the row's limit from here
        const int vis = qr.vis - (row + half * 4);
        if constexpr (MASKED) {
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[kb][i] = 32 * kb + 8 * (i / 4) + i % 4 < vis ? x[kb][i] * f[2 * kb + i / 8] : -INFINITY;
#pragma unroll
            for (int c = 0; c < 2 * NB; ++c) {
                f[c] = 1.f;
                vsc[c] = row + c * 16 < qr.vis ? vsc[c] : 0.f;      // only blocks that the row sees count, as there
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c) {
            float y = x[c >> 1][8 * (c & 1)];
#pragma unroll
            for (int i = 1; i < 8; ++i) y = fmaxf(y, x[c >> 1][8 * (c & 1) + i]);
            top = fmaxf(top, y * f[c]);
        }
        {
            auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
        }
        const int tile_exp = scale_exp(vsc), ve = max(vexp, MASKED ? tile_exp : (int)uniform((unsigned)tile_exp));
        if (__any(top > m + LAZY) || __any(ve > vexp)) {
            const float mn = fmaxf(m, top), alpha = exp2_hw(m - finite_or_zero(mn)), fo = times_pow2(alpha, vexp - ve);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= fo;
            sum *= alpha;
            m = mn;
            vexp = ve;
        }
        const float mz = finite_or_zero(m);
        h8_t ph[2 * NB], pl[2 * NB];
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c) {
            const float w = times_pow2(vsc[c], 15 - LAZY - vexp);
            float p[8], part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = exp2_hw(fmaf(x[c >> 1][8 * (c & 1) + i], f[c], -mz));
                part += p[i];
                p[i] *= w;
                // a masked weight is 0 whatever the scale is
                if constexpr (MASKED) p[i] = 16 * c + 8 * (i / 4) + i % 4 < vis ? p[i] : 0.f;
            }
            sum += part;
            weights_to_half(p, ph[c], pl[c]);
        }
        if (t + 1 < t_end) {
            store(t + 1, other);
            if (t + 2 < t_end) load(t + 2);
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int c = 0; c < 2 * NB; ++c) {
                const h8_t v = lds_read(v_get + c * 32 + dt * 32 * SM::V_ROW + buf);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, ph[c], o[dt], 0, 0, 0);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pl[c], o[dt], 0, 0, 0);
            }
        __syncthreads();
    };
    // tiles that every row sees, in pairs; then the others
    const int t_full = min(t_end, full / QT);
    int t = ta;
    for (; t + 2 <= t_full; t += 2) {
        round(t, std::integral_constant<unsigned, 0>{}, std::false_type{});
        round(t + 1, std::integral_constant<unsigned, SM::BUF>{}, std::false_type{});
    }
    for (; t < t_end; ++t) round(t, (t - ta) & 1 ? SM::BUF : 0u, std::true_type{});
    sum += __shfl_xor(sum, 32);
    int unit = vexp + LAZY - 15;
    if constexpr (KS == 2) {
        // the keys' halves meet: the second's result to the same lane of the first's wavefront
        static_assert(sizeof(QuantWideJoin<DH>) <= sizeof(sm));
        QuantWideJoin<DH> &jn = *(QuantWideJoin<DH> *)&sm;
        if (key32) {
#pragma unroll
            for (int u = 0; u < ND * 4; ++u) {
                qf4_t y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = times_pow2(o[u / 4][u % 4 * 4 + e], unit);
                jn.o[rows32][u][lane] = y;
            }
            jn.ml[rows32][lane] = make_float2(m, sum);
        }
        __syncthreads();
        if (key32) return;
        const float2 ml = jn.ml[rows32][lane];
        const float mm = fmaxf(m, ml.x), mz = finite_or_zero(mm);
        const float f0 = sum == 0.f ? 0.f : exp2f(m - mz), f1 = ml.y == 0.f ? 0.f : exp2f(ml.x - mz);    // 0: saw nothing
        sum = f0 * sum + f1 * ml.y;
        m = mm;
#pragma unroll
        for (int u = 0; u < ND * 4; ++u) {
            const qf4_t y = jn.o[rows32][u][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[u / 4][u % 4 * 4 + e] = f0 * times_pow2(o[u / 4][u % 4 * 4 + e], unit) + f1 * y[e];
        }
        unit = 0;
    }
    if (qr.vis < 0) return;
    // element i of o[dt]: dimension 32 dt + 8 (i / 4) + 4 half + i % 4 of row col
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t at = slot >= 0 ? (size_t)(blockIdx.x * 2 + slot) * RB + rows32 * 32 + col : (size_t)qr.row_of;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = times_pow2(o[dt][i + e], unit) * (slot >= 0 ? 1.f : inv);
            const size_t to = at * DH + dt * 32 + 2 * i + 4 * half;
            if (slot >= 0)
                *(qf4_t *)(a.ws_o + to) = qf4_t{y[0], y[1], y[2], y[3]};
            else
                store_row<4>(a.out, a.bf16, to, y);
        }
    if (half == 0) {
        if (slot >= 0)
            a.ws_ml[at] = make_float2(m, sum);
        else if (a.lse)
            a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * Q_LN2;
    }
}

template <int DH, int FMT, int KS>
__global__ __launch_bounds__(Q_THREADS, 2) void quant_wide_kernel(QuantAttend a)
{
    __shared__ QuantWideSmem<DH> sm;
    quant_parts(a, [&](const QuantSeq &sq, int b, int hd, int rb, int ta, int tb, int slot) {
        quant_wide_block<DH, FMT, KS>(a, sm, sq, b, hd, rb, ta, tb, slot);
    });
}

// Joins the pieces of a cache.  Which pieces of the workspace a block of rows has:
struct QuantPieces {
    unsigned w0, n;      // first work-group, pieces
    int RB;
    __device__ QuantPieces(const QuantAttend &a, const QuantShare &sh, const QuantSeq &sq, int b, unsigned hd, unsigned rb) : RB(a.RB)
    {
        const unsigned span = sh.span(sq), s0 = sh.before(a, b) + ((hd - b * sh.heads) * sq.nrb + rb) * span;
        w0 = sh.per == 1 ? s0 : s0 / sh.per;
        n = (sh.per == 1 ? s0 + span - 1 : (s0 + span - 1) / sh.per) - w0 + 1;
    }
    // row of piece p: slot 1 of its work-group for the first, 0 for the others
    __device__ size_t at(unsigned p, unsigned r) const { return (size_t)((w0 + p) * 2 + (p == 0)) * RB + (r & (RB - 1)); }
};

// Single tokens: a work-group per output row.  A lane has a piece's statistics; the wavefronts share the pieces' sums.  Makes
// the tiles' block sums shares of the whole as well.  576 rows of 7 pieces 5.4 us, 512 of 16 sequences 7.6: a launch and three
// dependent loads.
template <int DH>
__global__ __launch_bounds__(Q_THREADS) void quant_merge_kernel(QuantAttend a)
{
    constexpr int E = DH / 64;
    __shared__ float sm_o[4][DH];
    const QuantGeo &g = a.g;
    const unsigned row = blockIdx.x, hd = row / a.G, r = row - hd * a.G;      // n = 1
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = hd / (g.nl * g.H);
    const QuantSeq sq = quant_seq(a, b);
    if (sq.cnt == 0) return;
    QuantShare sh;
    sh.init(a, lane);
    const QuantPieces pc(a, sh, sq, b, hd, r >> a.rsh);
    float m = -INFINITY, sum = 0.f;
    if (pc.n == 1) {
        if (!a.mass) return;
        const float2 ml = a.ws_row[row];
        m = ml.x;
        sum = ml.y;
    } else {
        for (unsigned p0 = 0; p0 < pc.n; p0 += 64)
            if (p0 + lane < pc.n) m = fmaxf(m, a.ws_ml[pc.at(p0 + lane, r)].x);
        m = wave_maxf(m);
        const float mz = finite_or_zero(m);
        float x[E] = {};
        for (unsigned p0 = 0; p0 < pc.n; p0 += 64) {
            float f = 0.f;
            if (p0 + lane < pc.n) {
                const float2 ml = a.ws_ml[pc.at(p0 + lane, r)];
                if (ml.y != 0.f) f = exp2f(ml.x - mz);         // 0: the piece saw nothing
                sum += f * ml.y;
            }
            const int n = (int)min(64u, pc.n - p0);
#pragma unroll 4
            for (int p = wave; p < n; p += 4) {
                const float fp = lane_f(f, p);
                const float *o = a.ws_o + pc.at(p0 + p, r) * DH + lane * E;
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] += fp * o[e];
            }
        }
        sum = wave_sumf(sum);
#pragma unroll
        for (int e = 0; e < E; ++e) sm_o[wave][lane * E + e] = x[e];
        __syncthreads();
        if (tid < DH) {
            const float y = ((sm_o[0][tid] + sm_o[1][tid]) + (sm_o[2][tid] + sm_o[3][tid])) * (sum == 0.f ? 0.f : 1.f / sum);
            if (a.bf16)
                ((uint16_t *)a.out)[(size_t)row * DH + tid] = to_bf16(y);
            else
                ((float *)a.out)[(size_t)row * DH + tid] = y;
        }
        if (a.lse && tid == 0) a.lse[row] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * Q_LN2;
    }
    if (a.mass) mass_shares(a, row, sq.len, g.cap >> g.bsh, tid, Q_THREADS, m, sum == 0.f ? 0.f : 1.f / sum);
}

// Several tokens: a work-group per 16 rows of a head, sixteen threads a row.  32768 rows of two or three pieces 12.6 us, 46 MB.
template <int DH>
__global__ __launch_bounds__(Q_THREADS) void quant_merge_rows_kernel(QuantAttend a)
{
    constexpr int E = DH / 16;
    const unsigned groups = (a.R + 15) / 16, hd = blockIdx.x / groups, r0 = (blockIdx.x - hd * groups) * 16;
    const int b = hd / (a.g.nl * a.g.H);
    const QuantSeq sq = quant_seq(a, b);
    if ((int)r0 >= sq.cnt * a.G) return;
    QuantShare sh;
    sh.init(a, threadIdx.x & 63);
    const QuantPieces pc(a, sh, sq, b, hd, r0 >> a.rsh);
    const unsigned r = r0 + (threadIdx.x >> 4), d0 = (threadIdx.x & 15) * E;
    const QuantRow qr = quant_row(a, hd, r, sq.len, sq.cnt);
    if (pc.n == 1 || qr.vis < 0) return;
    float m = -INFINITY, sum = 0.f, x[E] = {};
#pragma unroll 4
    for (unsigned p = 0; p < pc.n; ++p) m = fmaxf(m, a.ws_ml[pc.at(p, r)].x);
    const float mz = finite_or_zero(m);
#pragma unroll 2
    for (unsigned p = 0; p < pc.n; ++p) {
        const float2 ml = a.ws_ml[pc.at(p, r)];
        const float f = ml.y == 0.f ? 0.f : exp2f(ml.x - mz);
        sum += f * ml.y;
        float o[E];
        __builtin_memcpy(o, __builtin_assume_aligned(a.ws_o + pc.at(p, r) * DH + d0, 16), sizeof(o));
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] += f * o[e];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= inv;
    store_row<E>(a.out, a.bf16, (size_t)qr.row_of * DH + d0, x);
    if (a.lse && d0 == 0) a.lse[qr.row_of] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * Q_LN2;
}

// ---- host ------------------------------------------------------------------------------------

thread_local char q_msg[256] = "no error";

wnw_status quant_fail(wnw_status st, const char *msg)
{
    strncpy(q_msg, msg, sizeof q_msg - 1);
    return st;
}
wnw_status quant_hip()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WNW_OK : quant_fail(WNW_ERR_HIP, hipGetErrorString(e));
}

bool aligned16(const void *p)
{
    return ((uintptr_t)p & 15) == 0;
}

wnw_status quant_config(const wnw_quant_config *c, int32_t first_layer, int32_t n_layers, int32_t n)
{
    if (!c) return quant_fail(WNW_ERR_INVALID, "NULL configuration");
    if (c->batch < 1 || c->layers < 1 || c->kv_heads < 1) return quant_fail(WNW_ERR_INVALID, "batch, layers and kv_heads must be at least 1");
    if (c->head_dim != 64 && c->head_dim != 128) return quant_fail(WNW_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (c->block != 16 && c->block != 32 && c->block != 64) return quant_fail(WNW_ERR_UNSUPPORTED, "block must be 16, 32 or 64");
    if (c->capacity < QT || c->capacity % QT) return quant_fail(WNW_ERR_INVALID, "capacity must be a positive multiple of 64");
    if (c->capacity > Q_MAX_CAP) return quant_fail(WNW_ERR_UNSUPPORTED, "capacity above 2^24 rows");
    if (c->format != WNW_QUANT_INT8 && c->format != WNW_QUANT_E4M3) return quant_fail(WNW_ERR_INVALID, "unknown format");
    if (c->flags & ~(uint32_t)WNW_F_OUT_BF16) return quant_fail(WNW_ERR_INVALID, "unknown flag bits");
    if (first_layer < 0 || n_layers < 1 || first_layer > c->layers - n_layers)
        return quant_fail(WNW_ERR_INVALID, "layers outside the cache's");
    if (n < 0 || n > c->capacity) return quant_fail(WNW_ERR_INVALID, "n outside 0 .. capacity");
    if ((int64_t)c->batch * n_layers > INT32_MAX / c->kv_heads) return quant_fail(WNW_ERR_UNSUPPORTED, "too many heads");
    return WNW_OK;
}

wnw_status quant_cache(const wnw_quant_cache *c)
{
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return quant_fail(WNW_ERR_INVALID, "NULL cache pointer");
    if (!aligned16(c->k) || !aligned16(c->v)) return quant_fail(WNW_ERR_INVALID, "cache bytes must be aligned to 16 bytes");
    if (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3) return quant_fail(WNW_ERR_INVALID, "scales must be aligned to 4 bytes");
    return WNW_OK;
}

QuantGeo quant_geo(const wnw_quant_config &c, const wnw_quant_cache &k, int32_t l0, int32_t nl)
{
    return QuantGeo{c.batch, c.layers, c.kv_heads, c.capacity, l0, nl, c.block == 16 ? 4 : c.block == 32 ? 5 : 6,
                    k.k, k.v, k.k_scale, k.v_scale};
}

// Tiles that n rows from any position on can touch.
int64_t touched_tiles(int32_t n)
{
    return ((int64_t)n + QT - 2) / QT + 1;
}

// Calls f with the configuration's head dimension and format as constants.
template <typename F>
void quant_dispatch(const wnw_quant_config &c, F f)
{
    using I0 = std::integral_constant<int, WNW_QUANT_INT8>;
    using I1 = std::integral_constant<int, WNW_QUANT_E4M3>;
    using D0 = std::integral_constant<int, 64>;
    using D1 = std::integral_constant<int, 128>;
    if (c.head_dim == 64)
        c.format == WNW_QUANT_INT8 ? f(D0{}, I0{}) : f(D0{}, I1{});
    else
        c.format == WNW_QUANT_INT8 ? f(D1{}, I0{}) : f(D1{}, I1{});
}

// Whether every block of rows gets a work-group of its own rather than blocks being cut into even parts and joined by a
// second launch.  Times in us, measured: a tile of a work-group that has its compute unit nearly alone (`tile`, four
// wavefronts in turn; `own`, as launched whole: eight of them, or four behind loads past the caches); a tile when the chip is
// full (`full`, a compute unit's time: the token kernels' bytes at 6.5 TB/s); and the join: its launch, which costs the host 3
// as well, the search for the parts (6) and, in the wide kernel, the parts' results to memory and back (8 for 512 of them).
// Measured whole and cut, tiles of one token, d = 128: 8 blocks of 12 9.3 and 10.5 us, of 24 13.2 and 12.3; 72 of 16 11.9 and
// 13.4, of 47 23.6 and 17.6; 128 of 32 18.4 and 20.8, of 63 29.4 and 30.5; 240 of 243 153 and 160, of 1423 848 and 866; d = 64:
// 8 of 16 7.2 and 8.8, of 47 13.0 and 10.3; 72 of 32 10.9 and 12.6; five tokens of four heads: 8 of 8 12.6 and 13.6, of 32 23.8
// and 19.1; 720 blocks of 147, 23 and 73 178 and 203; the wide kernel's blocks of 128 rows: 16 of 4 13.8 and 16.2, of 8 20.8 and
// 18.5, of 12 28.2 and 20.5; 64 of 8 21.8 and 22.9, of 32 64 and 38; 256 of 32 76 and 86, of 100 221 and 211, of 243 495 and 452;
// 512 of 63 233 and 251; 1024 of 63 455 and 483; of 64 rows: 8 of 5 11.5 and 13.7, of 16 22.6 and 15.2; 64 of 16 23.7 and 20.5; 240
// of 8 17.6 and 20.7, of 63 95 and 92, of 243 302 and 272.
// Of a batch only the longest length is known here, and every sequence is priced at it: a ragged batch whose longest sequence is
// walked whole waits for that sequence's blocks (16 ragged sequences of up to 20011 rows, d = 64, are cut, 30 us; 17 are
// whole, 71; 32 of up to 15512 rows, d = 128, 122 for 320 MB).
bool whole_blocks(int RB, int head_dim, int64_t blocks, int64_t tiles, bool eight, bool stream)
{
    const double b = blocks / 256.0, t = (double)tiles;
    if (RB > 32) {
        const double alone = RB == WIDE_ROWS ? 2.0 : 1.5, part = RB == WIDE_ROWS ? 1.8 : 1.3;
        const double whole = blocks <= 256 ? alone * t : 2 * part * t * (double)((blocks + 511) / 512);
        const double join = 6 + 8 * std::min(1.0, t * b / (2 * MIN_PIECE));
        return whole <= join + std::max(alone * MIN_PIECE, part * t * b);
    }
    const bool half = head_dim == 64;
    const double tile = half ? 0.3 : RB == 32 ? 0.6 : 0.45, full = half ? 0.32 : 0.63;
    const double own = eight ? (half ? 0.18 : RB == 32 ? 0.47 : 0.35) : stream && !half ? 0.55 : tile;
    return t * std::max(own, full * b) <= 6 + std::max(tile * MIN_PIECE, full * t * b);
}

// How an attention call runs: rows of a block, work-groups, loads past the caches; output rows; the workspace's arrays.
struct QuantPlan {
    int RB, W;       // RB 16, 32, 64 or 128
    bool whole, eight, stream;
    int64_t rows, o_bytes, ml_bytes, row_bytes, m_bytes;
    int64_t total() const { return o_bytes + ml_bytes + row_bytes + m_bytes; }
};
int64_t round16(int64_t x)
{
    return (x + 15) / 16 * 16;
}
QuantPlan quant_plan(const wnw_quant_config &c, int32_t n_layers, int32_t q_heads, int32_t n, int32_t max_len)
{
    const int64_t heads = (int64_t)c.batch * n_layers * c.kv_heads, R = (int64_t)q_heads / c.kv_heads * n;
    const int64_t len = max_len ? std::min(max_len, c.capacity) : c.capacity;
    QuantPlan p;
    // (only the token kernel makes masses)
    p.RB = n > 1 && R > 64 ? WIDE_ROWS : n > 1 && R > 32 ? WIDE_ROWS / 2 : R > 16 ? 32 : 16;
    const int64_t blocks = heads * ((R + p.RB - 1) / p.RB), tiles = (len + QT - 1) / QT * blocks;
    // Work-groups: one for every block of rows; or as many as the chip's 256 compute units hold at once, or as pieces of
    // MIN_PIECE tiles need.
    const int held = 256 * (c.head_dim == 64 && p.RB == 16 ? token_held<64, 1>() : 2);
    // Bytes that one pass reads once and the 256 MB of the last-level cache cannot keep for the next one
    p.stream = R <= p.RB && heads * len * c.head_dim * 2 > (256ll << 20);
    // Eight wavefronts instead of four for work-groups that have a compute unit each and a second round of tiles to share out
    // (128 blocks of 63 tiles 33.9 -> 29.4 us, 72 of 63 with d = 64 21.7 -> 17.0, 8 of 8 no difference).  Loads past the caches
    // that four wavefronts' instructions keep up with run 1 to 2 % faster with four (d = 128 and one block of 16 rows: 293.6
    // and 299.0 us for 30000 rows of 240 blocks; 32 rows 337 and 315, d = 64 149 and 145).
    p.eight = p.RB <= 32 && blocks <= 256 && len > 8 * QT && !(p.stream && p.RB == 16 && c.head_dim == 128);
    p.whole = whole_blocks(p.RB, c.head_dim, blocks, (len + QT - 1) / QT, p.eight, p.stream);
    p.eight = p.eight && p.whole;
    p.W = (int)std::max<int64_t>(1, p.whole ? blocks : std::min<int64_t>(held, tiles / MIN_PIECE + blocks));
    p.rows = heads * R;
    p.o_bytes = p.whole ? 0 : (int64_t)p.W * 2 * p.RB * c.head_dim * 4;
    p.ml_bytes = p.whole ? 0 : (int64_t)p.W * 2 * p.RB * 8;
    p.row_bytes = n == 1 && !p.whole ? round16(p.rows * 8) : 0;
    p.m_bytes = n == 1 ? round16(p.rows * (c.capacity / QT) * 4) : 0;
    return p;
}

template <int DH, int FMT, int MT>
void launch_few(const QuantPlan &p, const QuantAttend &a, hipStream_t st)
{
    constexpr bool both = DH == 64 || MT == 2;
    auto *k = p.eight ? (p.stream ? quant_token_kernel<DH, FMT, MT, both, 8> : quant_token_kernel<DH, FMT, MT, false, 8>)
                      : (p.stream ? quant_token_kernel<DH, FMT, MT, true, 4> : quant_token_kernel<DH, FMT, MT, false, 4>);
    hipLaunchKernelGGL(k, dim3(p.W), dim3(p.eight ? 512 : 256), 0, st, a);
}
template <int DH, int FMT>
void launch_token(const QuantPlan &p, const QuantAttend &a, hipStream_t st)
{
    if (p.RB == WIDE_ROWS)
        hipLaunchKernelGGL((quant_wide_kernel<DH, FMT, 1>), dim3(p.W), dim3(Q_THREADS), 0, st, a);
    else if (p.RB == WIDE_ROWS / 2)
        hipLaunchKernelGGL((quant_wide_kernel<DH, FMT, 2>), dim3(p.W), dim3(Q_THREADS), 0, st, a);
    else if (p.RB == 32)
        launch_few<DH, FMT, 2>(p, a, st);
    else
        launch_few<DH, FMT, 1>(p, a, st);
}

wnw_status quant_heads(const wnw_quant_config &c, int32_t n_layers, int32_t q_heads, int32_t n, int32_t max_len)
{
    if (q_heads < c.kv_heads || q_heads % c.kv_heads) return quant_fail(WNW_ERR_INVALID, "q_heads must be a multiple of kv_heads");
    if (max_len < 0) return quant_fail(WNW_ERR_INVALID, "negative max_len");
    if ((int64_t)c.batch * n_layers * q_heads > (n > 1 ? INT32_MAX / n : Q_MAX_GROUPS))
        return quant_fail(WNW_ERR_UNSUPPORTED, "too many query rows");
    // the line of tiles is counted in 32 bits
    const int64_t blocks = ((int64_t)q_heads / c.kv_heads * n + 15) / 16 * c.batch * n_layers * c.kv_heads;
    if (blocks > Q_MAX_GROUPS || blocks > INT32_MAX / (c.capacity / QT)) return quant_fail(WNW_ERR_UNSUPPORTED, "too many tiles for one call");
    return WNW_OK;
}

}  // namespace

}  // namespace wnw

using namespace wnw;

extern "C" {

const char *wnw_quant_last_error(void)
{
    return q_msg;
}

wnw_status wnw_quant_write(const wnw_quant_config *cfg, const wnw_quant_cache *cache, int32_t first_layer, int32_t n_layers,
                           int32_t n, const void *k_dev, const void *v_dev, const int32_t *pos_dev, const int32_t *count_dev,
                           void *hip_stream)
{
    wnw_status st = quant_config(cfg, first_layer, n_layers, n);
    if (st == WNW_OK) st = quant_cache(cache);
    if (st != WNW_OK) return st;
    if (n == 0) return WNW_OK;
    if (!k_dev || !v_dev || !pos_dev) return quant_fail(WNW_ERR_INVALID, "NULL pointer");
    if (!aligned16(k_dev) || !aligned16(v_dev)) return quant_fail(WNW_ERR_INVALID, "rows must be aligned to 16 bytes");
    const int64_t tiles = touched_tiles(n), groups = 2 * tiles * cfg->batch * n_layers * cfg->kv_heads;
    if (groups > Q_MAX_GROUPS) return quant_fail(WNW_ERR_UNSUPPORTED, "too many rows for one call");
    const QuantGeo g = quant_geo(*cfg, *cache, first_layer, n_layers);
    quant_dispatch(*cfg, [&](auto d, auto f) {
        constexpr int DH = decltype(d)::value, FMT = decltype(f)::value;
        const uint16_t *k = (const uint16_t *)k_dev, *v = (const uint16_t *)v_dev;
        const int heads = cfg->batch * n_layers * cfg->kv_heads;
        if (n <= APPEND_ROWS)
            hipLaunchKernelGGL((quant_append_kernel<DH, FMT>), dim3((unsigned)(heads + 1) / 2), dim3(Q_THREADS), 0, (hipStream_t)hip_stream, g,
                               n, 2 * heads, k, v, pos_dev, count_dev);
        else
            hipLaunchKernelGGL((quant_write_kernel<DH, FMT>), dim3((unsigned)groups), dim3(Q_THREADS), 0, (hipStream_t)hip_stream, g, n,
                               (int)tiles, k, v, pos_dev, count_dev);
    });
    return quant_hip();
}

wnw_status wnw_quant_read(const wnw_quant_config *cfg, const wnw_quant_cache *cache, int32_t first_layer, int32_t n_layers,
                          int32_t n, void *k_out, void *v_out, const int32_t *pos_dev, const int32_t *count_dev, void *hip_stream)
{
    wnw_status st = quant_config(cfg, first_layer, n_layers, n);
    if (st == WNW_OK) st = quant_cache(cache);
    if (st != WNW_OK) return st;
    if (n == 0 || (!k_out && !v_out)) return WNW_OK;
    if (!pos_dev) return quant_fail(WNW_ERR_INVALID, "NULL pointer");
    if (!aligned16(k_out) || !aligned16(v_out)) return quant_fail(WNW_ERR_INVALID, "outputs must be aligned to 16 bytes");
    const int64_t tiles = touched_tiles(n), groups = (k_out && v_out ? 2 : 1) * tiles * cfg->batch * n_layers * cfg->kv_heads;
    if (groups > Q_MAX_GROUPS) return quant_fail(WNW_ERR_UNSUPPORTED, "too many rows for one call");
    const QuantGeo g = quant_geo(*cfg, *cache, first_layer, n_layers);
    const bool bf16 = cfg->flags & WNW_F_OUT_BF16;
    quant_dispatch(*cfg, [&](auto d, auto f) {
        constexpr int DH = decltype(d)::value, FMT = decltype(f)::value;
        hipLaunchKernelGGL((bf16 ? quant_read_kernel<DH, FMT, true> : quant_read_kernel<DH, FMT, false>), dim3((unsigned)groups),
                           dim3(Q_THREADS), 0, (hipStream_t)hip_stream, g, n, (int)tiles, k_out, v_out, pos_dev, count_dev);
    });
    return quant_hip();
}

wnw_status wnw_quant_attend_workspace(const wnw_quant_config *cfg, int32_t n_layers, int32_t q_heads, int32_t n, int32_t max_len,
                                      size_t *bytes)
{
    wnw_status st = quant_config(cfg, 0, n_layers, n);
    if (st == WNW_OK) st = quant_heads(*cfg, n_layers, q_heads, n, max_len);
    if (st != WNW_OK) return st;
    if (!bytes) return quant_fail(WNW_ERR_INVALID, "NULL pointer");
    *bytes = (size_t)quant_plan(*cfg, n_layers, q_heads, n, max_len).total();
    return WNW_OK;
}

wnw_status wnw_quant_attend(const wnw_quant_config *cfg, const wnw_quant_cache *cache, int32_t first_layer, int32_t n_layers,
                            int32_t q_heads, int32_t n, const void *q_dev, const int32_t *len_dev, const int32_t *count_dev,
                            void *out_dev, float *lse_dev, float *mass_dev, int32_t max_len, void *workspace,
                            size_t workspace_bytes, void *hip_stream)
{
    wnw_status st = quant_config(cfg, first_layer, n_layers, n);
    if (st == WNW_OK) st = quant_cache(cache);
    if (st == WNW_OK) st = quant_heads(*cfg, n_layers, q_heads, n, max_len);
    if (st != WNW_OK) return st;
    if (mass_dev && n > 1) return quant_fail(WNW_ERR_INVALID, "block masses are of single tokens (n = 1)");
    if (n == 0) return WNW_OK;
    if (!q_dev || !len_dev || !out_dev) return quant_fail(WNW_ERR_INVALID, "NULL pointer");
    if (!aligned16(q_dev) || !aligned16(out_dev)) return quant_fail(WNW_ERR_INVALID, "queries and outputs must be aligned to 16 bytes");
    const QuantPlan p = quant_plan(*cfg, n_layers, q_heads, n, max_len);
    if (p.total() && (!workspace || !aligned16(workspace) || workspace_bytes < (size_t)p.total()))
        return quant_fail(WNW_ERR_INVALID, "workspace missing, too small or not aligned to 16 bytes");
    const int G = q_heads / cfg->kv_heads, R = G * n;
    char *ws = (char *)workspace;
    QuantAttend a = {quant_geo(*cfg, *cache, first_layer, n_layers), G, n, R, p.W, p.RB, p.RB == 16 ? 4 : p.RB == 32 ? 5 : p.RB == 64 ? 6 : 7,
                     cfg->flags & WNW_F_OUT_BF16 ? 1 : 0, p.whole ? (R + p.RB - 1) / p.RB : 0, 1.f / p.W, (const uint16_t *)q_dev, len_dev, count_dev, out_dev,
                     lse_dev, mass_dev, (float *)ws, (float2 *)(ws + p.o_bytes),
                     (float2 *)(ws + p.o_bytes + p.ml_bytes), (float *)(ws + p.o_bytes + p.ml_bytes + p.row_bytes),
                     Q_LOG2E / sqrtf((float)cfg->head_dim)};
    quant_dispatch(*cfg, [&](auto d, auto f) {
        constexpr int DH = decltype(d)::value, FMT = decltype(f)::value;
        launch_token<DH, FMT>(p, a, (hipStream_t)hip_stream);
        if (p.whole) return;
        if (n == 1)
            hipLaunchKernelGGL((quant_merge_kernel<DH>), dim3((unsigned)p.rows), dim3(Q_THREADS), 0, (hipStream_t)hip_stream, a);
        else
            hipLaunchKernelGGL((quant_merge_rows_kernel<DH>), dim3((unsigned)(p.rows / R * ((R + 15) / 16))), dim3(Q_THREADS), 0,
                               (hipStream_t)hip_stream, a);
    });
    return quant_hip();
}

}  // extern "C"
