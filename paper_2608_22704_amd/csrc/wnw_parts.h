// What the attention kernels over caches share: steps across a wavefront's lanes, how the tiles of a batch of any lengths are
// shared out to work-groups, and which results are joined afterwards.
//
// A, the arguments of such a kernel, has: g with B sequences and nl * H KV-heads a sequence; len and count (device, see below; count
// may be null); cap, the most rows of a sequence; tiles_of(rows); n tokens, G q-heads per KV-head, R = n G query rows of a KV-head (row
// r is token r / G, q-head r % G), in blocks of RB = 2^rsh; W work-groups and inv_w = 1 / W; nrb > 0: a work-group for
// every block of rows, nrb of them a head.  group(): the work-group's number, 0 .. W - 1, in the order in which parts are dealt
// out (and in which the workspace has them).  whole_block(hd, rb): the block of a work-group where nrb > 0.  BLOCK_COST: see below.
#pragma once

#include "wnw_lds.h"

#include <math.h>

namespace wnw {

__device__ inline int clamp_to(int x, int hi)
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

// As load_to_lds, past the caches that a stream does not fit.
__device__ inline void stream_to_lds(const void *base, unsigned off, unsigned lds)
{
    __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base) : "m0", "memory");
}

// The kernel's arguments once more, as memory: what only its last part needs is loaded there, and does not take scalar
// registers from the start (fetching instructions is what a short call waits for, and spills are instructions).
template <typename A>
__device__ inline const A &late_args()
{
    auto *p = (const __attribute__((address_space(4))) A *)__builtin_amdgcn_kernarg_segment_ptr();
    __asm__ volatile("" : "+s"(p));
    return *(const A *)p;
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

// Work of a batch: every block of RB query rows of every head has its sequence's tiles (one at least, so that an
// empty sequence's outputs are written).  W work-groups share them, whatever the lengths are, in one of two ways:
//   pieces  a block's tiles are cut into pieces of at most `pp` tiles, a work-group each;
//   line    all tiles in a line, in the order sequence, head, block of rows, tile, are cut into W equal parts (pp = 0), so that a
//           work-group's part may end one block and begin another.  In front of its tiles a block has A::BLOCK_COST places
//           that stand for its start, so that many short blocks do not count as little.
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

struct PartSeq {
    int len, cnt, tiles, nrb;   // rows, tokens of this call, tiles and blocks of rows of a head (0: none)
};
template <typename A>
__device__ inline PartSeq part_seq(const A &a, int b)
{
    PartSeq q = {0, 0, 1, 0};
    if (b < a.g.B) {
        q.len = clamp_to(a.len[b], a.cap());
        q.cnt = a.count ? clamp_to(a.count[b], a.n) : a.n;
        q.tiles = max(1, a.tiles_of(q.len));
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
template <typename A>
struct PartShare {
    int heads, lane;
    int pp;              // tiles of a piece, or 0: the line
    unsigned per;        // items per work-group (tiles of the line, or 1 piece)
    unsigned total;      // items
    PartSeq mine;       // sequence `lane`

    __device__ PartSeq seq(const A &a, int b0) const { return b0 == 0 ? mine : part_seq(a, b0 + lane); }
    // items of a block of rows
    __device__ unsigned span(const PartSeq &q) const { return pp ? (unsigned)div24(q.tiles + pp - 1, pp) : (unsigned)(q.tiles + A::BLOCK_COST); }
    __device__ unsigned work(const PartSeq &q) const { return span(q) * (unsigned)(q.nrb * heads); }

    __device__ void init(const A &a, int lane_)
    {
        heads = a.g.nl * a.g.H, lane = lane_, pp = 0;
        unsigned t = 0, units = 0, most = 0;
        if (a.g.B == 1) {       // (all of it scalar, and no other instructions to fetch)
            mine = part_seq(a, 0);
            t = work(mine), units = (unsigned)(mine.nrb * heads), most = mine.nrb ? (unsigned)mine.tiles : 0u;
        } else {
            mine = part_seq(a, lane);
            for (int b0 = 0; b0 < a.g.B; b0 += 64) {
                const PartSeq q = seq(a, b0);
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
            const unsigned p = min(max(at_least(t - units * A::BLOCK_COST, __builtin_amdgcn_rcpf((float)(a.W - units))), (unsigned)MIN_PIECE), most);
            if (p && piece_len((int)most, (int)p) <= (int)per + (A::BLOCK_COST ? 0 : PIECE_COST)) {
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
    __device__ int find(const A &a, unsigned f, unsigned &start, PartSeq &sq) const
    {
        if (a.g.B == 1) {
            start = 0;
            sq = {(int)uniform(mine.len), (int)uniform(mine.cnt), (int)uniform(mine.tiles), (int)uniform(mine.nrb)};
            return 0;
        }
        unsigned base = 0;
        for (int b0 = 0;; b0 += 64) {
            const PartSeq q = seq(a, b0);
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
    __device__ unsigned before(const A &a, int end) const
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

struct PartRow {
    int row_of;      // index into [B][nl][H_q][n] of row r
    int vis;         // cache rows it sees; -1: not a row of this call
};
template <typename A>
__device__ inline PartRow part_row(const A &a, int hd, int r, int len, int cnt)
{
    const int i = a.n == 1 ? 0 : r / a.G, j = r - i * a.G;
    PartRow q;
    q.row_of = (hd * a.G + j) * a.n + i;      // hd = (b * nl + l) * H + h
    q.vis = r < a.R && i < cnt ? max(0, min(len, len - cnt + i + 1)) : -1;
    return q;
}

// Runs f(sequence, b, head, block of rows, first tile, end tile, slot) for the work-group's part of a batch.
template <typename A, typename F>
__device__ inline void run_parts(const A &a, F f)
{
    PartShare<A> sh;
    PartSeq sq;
    int b = 0, hd, rb, ta = 0, tb;
    unsigned i = 0, i1 = 0, start = 0;
    auto item = [&]() {
        const unsigned off = i - start, span = uniform(sh.span(sq));
        const unsigned unit = span == 1 ? off : sh.pp ? (unsigned)div24((int)off, (int)span) : off / span, at = off - unit * span;
        ta = (int)at;
        tb = (int)min(span, at + (i1 - i));
        i += tb - ta;
        if (A::BLOCK_COST && !sh.pp) ta = max(0, ta - A::BLOCK_COST), tb = max(0, tb - A::BLOCK_COST);
        if (sh.pp) {
            const int len = PartShare<A>::piece_len(sq.tiles, sh.pp);
            ta = min(sq.tiles, (int)at * len);
            tb = min(sq.tiles, ta + len);
        }
        hd = sq.nrb == 1 ? (int)unit : (int)unit / sq.nrb;
        rb = (int)unit - hd * sq.nrb;
        hd = (int)uniform(hd + b * sh.heads), rb = (int)uniform(rb), ta = (int)uniform(ta), tb = (int)uniform(tb);
    };
    if (a.nrb > 0) {
        a.whole_block(hd, rb);
        if (a.g.B > 1) b = hd / (a.g.nl * a.g.H);
        sq = part_seq(a, b);
        if (rb >= sq.nrb) return;
        tb = sq.tiles;
    } else {
        sh.init(a, threadIdx.x & 63);
        i = a.group() * sh.per;
        if (i >= sh.total) return;
        i1 = min(i + sh.per, sh.total);
        b = sh.find(a, i, start, sq);
        item();
    }
    for (;;) {
        if (!A::BLOCK_COST || tb > ta) f(sq, b, hd, rb, ta, tb, ta > 0 ? 0 : tb < sq.tiles ? 1 : -1);
        if (i >= i1) return;
        if (i - start >= sh.work(sq)) b = sh.find(a, i, start, sq);
        item();
        __syncthreads();
    }
}

// Joins the pieces of a cache.  Which pieces of the workspace a block of rows has:
template <typename A>
struct PartPieces {
    unsigned w0, n;      // first work-group, pieces
    int RB;
    __device__ PartPieces(const A &a, const PartShare<A> &sh, const PartSeq &sq, int b, unsigned hd, unsigned rb) : RB(a.RB)
    {
        const unsigned span = sh.span(sq), s0 = sh.before(a, b) + ((hd - b * sh.heads) * sq.nrb + rb) * span;
        w0 = sh.per == 1 ? s0 : (s0 + A::BLOCK_COST) / sh.per;
        n = (sh.per == 1 ? s0 + span - 1 : (s0 + span - 1) / sh.per) - w0 + 1;
    }
    // row of piece p: slot 1 of its work-group for the first, 0 for the others
    __device__ size_t at(unsigned p, unsigned r) const { return (size_t)((w0 + p) * 2 + (p == 0)) * RB + (r & (RB - 1)); }
};

}  // namespace wnw
