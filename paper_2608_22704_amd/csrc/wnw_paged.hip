// A paged KV cache in bf16: appending rows with the rotation of their positions, attention over the pages for single tokens,
// drafts, their trees and prompts, and moving the rows of accepted tokens.  Layout and definitions as in wnw.h.
//
//   paged_append_kernel  new rows of K and V to their pages and queries to their place, rotated on the way
//   paged_keep_kernel    accepted rows to the end of their sequence, a wavefront per head's K or V
//   paged_token_kernel   attention in blocks of 16 or 32 query rows of a KV-head, every wavefront with tiles of its own
//   paged_wide_kernel    attention in blocks of 64, 128 or 256 query rows, whose wavefronts share tiles
//   paged_join_kernel    joins the parts of a cache that work-groups shared
#include "wnw.h"
#include "wnw_internal.h"
#include "wnw_parts.h"

#include <math.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

namespace wnw {

namespace {

constexpr int P_THREADS = 256;
constexpr int P_MAX_CAP = 1 << 24;
constexpr int64_t P_MAX_GROUPS = 0xffffffffll / P_THREADS;   // a launch has fewer than 2^32 threads
constexpr float P_LOG2E = 1.4426950408889634f;
constexpr float P_LN2 = 0.6931471805599453f;

typedef float pf4_t __attribute__((ext_vector_type(4)));
typedef unsigned pu2_t __attribute__((ext_vector_type(2)));
typedef unsigned pu4_t __attribute__((ext_vector_type(4)));
typedef short ps4_t __attribute__((ext_vector_type(4)));

// The pages and the layers of them that a call handles.
struct PagedGeo {
    int B, L, H, l0, nl;
    int pages, width, psh;    // pages of the buffers and of a sequence, log2 of a page's rows
    uint16_t *k, *v;
    const int32_t *table;
    __host__ __device__ int cap() const { return width << psh; }
    // first row, in rows of d elements, that page `id` has for layer l0 + l and KV-head h
    __device__ size_t page_row(int id, int l, int h) const { return (((size_t)id * L + l0 + l) * H + h) << psh; }
    __device__ bool has(int id) const { return (unsigned)id < (unsigned)pages; }
};

__device__ inline uint16_t to_bf16(float f)
{
    return __builtin_bit_cast(uint16_t, (__bf16)f);   // nearest, ties to even
}
__device__ inline float bf16_at(pu4_t u, int e)
{
    return __uint_as_float(e & 1 ? u[e >> 1] & 0xffff0000u : u[e >> 1] << 16);
}

// ---- appending -------------------------------------------------------------------------------

struct PagedAppend {
    PagedGeo g;
    int Hq, n, tiles, split;     // tiles: groups of tokens; split: work-groups that share a layer's vectors
    int dim, vectors;            // vectors of a token and layer: K and V of every KV-head, then the queries
    float amplitude;
    const float *freq;
    const uint16_t *kn, *vn, *q;
    uint16_t *q_out;
    const int32_t *at, *count, *position;
};

// How a pair's two elements lie.
enum { TURN_NONE, TURN_PAIRS, TURN_HALVES, TURN_HALVES_ODD };

// A lane has 16 bytes (eight elements) of a vector: neighbours d / 8 lanes one vector, and the work-group TT tokens' vectors of
// HH heads at a time, going through the layer's heads with the angles of its lanes in registers, which depend on token and element
// alone (in a work-group per head the 64-bit angles, cosines and sines would be as much work as the bytes).  An element's partner is in
// the lane itself (pairs) or comes from the lane that has it, halves of a multiple of eight elements by four moves, others by two
// for each element.
// Bound by memory, which it reads and writes once: 7756 rows of 36 layers with 16 q-heads and 2 KV-heads, 2.86 GB, take 511 us, 5.6 TB/s
// (540 with one vector of a lane under way instead of UNROLL).  A single token is bound by the
// launch and one chain of table, positions and rows: all of 30 layers with 32 and 8 heads 5.6 us on the GPU.
template <int DH, int TURN>
__global__ __launch_bounds__(P_THREADS) void paged_append_kernel(PagedAppend a, int TT)
{
    constexpr int UN = DH / 8, SLOTS = P_THREADS / UN, UNROLL = TURN == TURN_HALVES_ODD ? 1 : 4;
    const PagedGeo &g = a.g;
    const int HH = SLOTS / TT, tid = threadIdx.x, u = tid % UN, slot = tid / UN, lane = tid & 63;
    int item = blockIdx.x;
    const int part = item % a.split;
    item /= a.split;
    const int tile = item % a.tiles;
    item /= a.tiles;
    const int l = item % g.nl, b = item / g.nl;
    const int i = tile * TT + slot % TT, cnt = a.count ? clamp_to(a.count[b], a.n) : a.n;
    if (tile * TT >= cnt) return;
    const bool live = i < cnt;
    const int at = clamp_to(a.at[b], g.cap()), row = at + i;
    int id = -1;
    if (live && row < g.cap()) id = g.table[(size_t)b * g.width + (row >> g.psh)];
    const bool place = g.has(id);
    // the lane's angles
    float cs[8], sn[8];
    const int half = a.dim >> 1;
    if constexpr (TURN != TURN_NONE) {
        const double pos = a.position && live ? (double)a.position[(size_t)b * a.n + i] : (double)row;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int x = u * 8 + e;
            if (TURN == TURN_PAIRS && (e & 1)) {
                cs[e] = cs[e - 1], sn[e] = -sn[e - 1];
                continue;
            }
            cs[e] = 1.f, sn[e] = 0.f;
            if (x < a.dim) {
                const int pair = TURN == TURN_PAIRS ? x >> 1 : x < half ? x : x - half;
                // turns, and without the whole ones: the product of position and frequency is exact in a double below 2^29
                const double turns = pos * (double)a.freq[pair] * 0.15915494309189535;
                const float rest = (float)(turns - rint(turns));
                float s, c;
                sincospif(2.f * rest, &s, &c);
                cs[e] = c * a.amplitude;
                sn[e] = s * a.amplitude;
                if (TURN == TURN_PAIRS || x < half) sn[e] = -sn[e];
            }
        }
    }
    // vectors of K, V and q in turn, UNROLL at a time, so that as many loads are under way
    const int kv = a.kn ? 2 * g.H : 0, step = a.split * HH;
    const size_t in_page = row & ((1 << g.psh) - 1), first = ((size_t)b * g.nl + l);
    auto from = [&](int v) {
        const bool is_q = v >= kv;
        const int h = is_q ? v - kv : v >= g.H ? v - g.H : v;
        return (is_q ? a.q : v >= g.H ? a.vn : a.kn) + ((first * (is_q ? a.Hq : g.H) + h) * a.n + i) * DH + u * 8;
    };
    auto to = [&](int v) {
        if (v >= kv) return a.q_out + ((first * a.Hq + (v - kv)) * a.n + i) * DH + u * 8;
        return (v >= g.H ? g.v : g.k) + (g.page_row(id, l, v >= g.H ? v - g.H : v) + in_page) * DH + u * 8;
    };
    for (int v0 = part * HH + slot / TT; v0 < a.vectors; v0 += UNROLL * step) {
        pu4_t xs[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int v = v0 + k * step;
            xs[k] = pu4_t{0, 0, 0, 0};
            if (v < a.vectors && (v >= kv ? live : place)) xs[k] = __builtin_nontemporal_load((const pu4_t *)from(v));
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int v = v0 + k * step;
            pu4_t x = xs[k];
            const bool is_v = v >= g.H && v < kv;
            if constexpr (TURN != TURN_NONE) {
                pu4_t o = x;     // partners
                if constexpr (TURN == TURN_PAIRS) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = x[e] << 16 | x[e] >> 16;
                } else if constexpr (TURN == TURN_HALVES) {
                    const int hu = half >> 3, other = u < hu ? u + hu : u < 2 * hu ? u - hu : u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = (unsigned)__shfl((int)x[e], lane - u + other);
                } else {
                    const int up = half & 7, down = 8 - up, hu = half >> 3;      // half = 8 hu + up
                    uint16_t y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        // from u + hu (+ 1) or from u - hu (- 1); the words to send are the same for all lanes
                        const int e0 = (e + up) & 7, e1 = (e + down) & 7;
                        unsigned w0 = x[0], w1 = x[0];
#pragma unroll
                        for (int j = 1; j < 4; ++j) {
                            w0 = e0 >> 1 == j ? x[j] : w0;
                            w1 = e1 >> 1 == j ? x[j] : w1;
                        }
                        const int l0 = u + hu + (e + up >= 8), l1 = u - hu - (e < up);
                        const unsigned g0 = (unsigned)__shfl((int)w0, lane - u + min(max(l0, 0), UN - 1)),
                                       g1 = (unsigned)__shfl((int)w1, lane - u + min(max(l1, 0), UN - 1));
                        const bool low = u * 8 + e < half;
                        const unsigned w = low ? g0 : g1;
                        y[e] = (uint16_t)((low ? e0 : e1) & 1 ? w >> 16 : w);
                    }
                    __builtin_memcpy(&o, y, sizeof(o));
                }
                if (!is_v) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y0 = fmaf(bf16_at(o, 2 * e), sn[2 * e], bf16_at(x, 2 * e) * cs[2 * e]),
                                    y1 = fmaf(bf16_at(o, 2 * e + 1), sn[2 * e + 1], bf16_at(x, 2 * e + 1) * cs[2 * e + 1]);
                        const unsigned r0 = u * 8 + 2 * e < a.dim ? to_bf16(y0) : x[e] & 0xffffu,
                                       r1 = u * 8 + 2 * e + 1 < a.dim ? to_bf16(y1) : x[e] >> 16;
                        x[e] = r0 | r1 << 16;
                    }
                }
            }
            if (v < a.vectors && (v >= kv ? live : place)) __builtin_nontemporal_store(x, (pu4_t *)to(v));
        }
    }
}

// ---- keeping ---------------------------------------------------------------------------------

// A wavefront has a head's K or V, so that no other has the rows that it reads and writes.  A path ascends, so that row base + i is no
// source of a later entry, and the rows of one step are read before any of them is written.  Bound by latency (path, table entry, row): a
// path of 64 tokens of which three stand in one layer of 8 KV-heads takes 3.1 us on the GPU, eight sequences of 30 such layers with up to eight
// 4.7; a launch with nothing to do takes 2.
template <int DH>
__global__ __launch_bounds__(P_THREADS) void paged_keep_kernel(PagedGeo g, int n, int items, const int32_t *__restrict__ base_dev,
                                                               const int32_t *__restrict__ path_dev,
                                                               const int32_t *__restrict__ count_dev)
{
    constexpr int UN = DH / 8, ROWS = 64 / UN, STEP = 4;
    const int item = blockIdx.x * (P_THREADS / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (item >= items) return;
    const bool is_v = item & 1;
    const int hd = item >> 1, b = hd / (g.nl * g.H), lh = hd - b * g.nl * g.H, l = lh / g.H, h = lh - l * g.H;
    const int cap = g.cap(), base = clamp_to(base_dev[b], cap);
    const int32_t *path = path_dev + (size_t)b * n, *table = g.table + (size_t)b * g.width;
    int cnt = count_dev ? clamp_to(count_dev[b], n) : n;
    for (int i0 = 0; i0 < cnt; i0 += 64) {
        const int i = i0 + lane;
        bool ends = false;
        if (i < cnt) ends = path[i] < 0 || path[i] >= cap - base || (i > 0 && path[i] <= path[i - 1]);
        const unsigned long long some = __ballot(ends);
        if (some) cnt = i0 + __builtin_ctzll(some);
    }
    uint16_t *pool = is_v ? g.v : g.k;
    const int u = lane % UN, r = lane / UN, mask = (1 << g.psh) - 1;
    for (int i0 = 0; i0 < cnt; i0 += ROWS * STEP) {
        pu4_t x[STEP];
        uint16_t *to[STEP];
#pragma unroll
        for (int j = 0; j < STEP; ++j) {
            const int i = i0 + j * ROWS + r;
            to[j] = nullptr;
            if (i >= cnt || path[i] == i) continue;
            const int from = base + path[i], into = base + i, id0 = table[from >> g.psh], id1 = table[into >> g.psh];
            if (!g.has(id0) || !g.has(id1)) continue;
            x[j] = *(const pu4_t *)(pool + (g.page_row(id0, l, h) + (from & mask)) * DH + u * 8);
            to[j] = pool + (g.page_row(id1, l, h) + (into & mask)) * DH + u * 8;
        }
#pragma unroll
        for (int j = 0; j < STEP; ++j)
            if (to[j]) *(pu4_t *)to[j] = x[j];
    }
}

// ---- attention -------------------------------------------------------------------------------

struct PagedAttend {
    PagedGeo g;
    int G, n, R;               // q-heads per KV-head, tokens, rows G * n of a KV-head: row r is token r / G, q-head r % G
    int W, RB, rsh;            // work-groups that share the batch's tiles, rows of a block and their log2
    int tsh;                   // log2 of the cache rows of a tile
    int bf16;                  // outputs are bf16: the fp32 results, rounded as they are stored
    int nrb;                   // > 0: a work-group per block of rows, nrb blocks a head, nothing to join
    float inv_w;               // 1 / W
    const uint16_t *q;
    const int32_t *len, *count;
    const unsigned long long *mask;
    void *out;
    float *lse;
    float *ws_o;               // [W][2][RB][d]: sums of weights times values of a block of rows over a piece of its cache
    float2 *ws_ml;             // [W][2][RB]: the piece's maximum (base 2) and sum of weights
    float scale;               // log2(e) / sqrt(d)
    static constexpr int BLOCK_COST = 8;      // a block's start in tiles' times
    __device__ int cap() const { return g.cap(); }
    // Work-groups go to the eight dies in turn; those that follow each other here are on one die, whose cache then serves the blocks of
    // rows of one head.
    __device__ unsigned group() const
    {
        const unsigned die = blockIdx.x & 7, each = (unsigned)W >> 3, more = (unsigned)W & 7;
        return die * each + min(die, more) + (blockIdx.x >> 3);
    }
    // Which block a work-group has where blocks are whole.  Without a mask later tokens see more rows, so the last ones of a head begin, and
    // the dies get as many of every length: whole heads each, one after the other, after those heads that are left over, whose blocks go to
    // the dies in turn (a prompt of 7756 tokens, 32 heads over 8: 976 us in the order of heads and blocks, 850 so; 16 over 2: 674 and 436).
    __device__ void whole_block(int &hd, int &rb) const
    {
        if (nrb == 1) {
            hd = (int)group(), rb = 0;
            return;
        }
        const int heads = g.B * g.nl * g.H, over = heads & 7, x = (int)blockIdx.x - over * nrb;
        if (x < 0) {
            rb = (int)blockIdx.x / over;
            hd = heads - over + (int)blockIdx.x - rb * over;
        } else {
            hd = (x >> 3) / nrb;
            rb = (x >> 3) - hd * nrb;
            hd += (x & 7) * (heads >> 3);
        }
        rb = nrb - 1 - rb;
    }
    __device__ int tiles_of(int rows) const { return (rows + (1 << tsh) - 1) >> tsh; }
};

template <int E>
__device__ inline void store_out(void *out, bool bf16, size_t elem, const float (&x)[E])
{
    if (bf16) {
        uint16_t u[E];
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = to_bf16(x[e]);
        __builtin_memcpy(__builtin_assume_aligned((uint16_t *)out + elem, E * 2), u, sizeof(u));
    } else
        __builtin_memcpy(__builtin_assume_aligned((float *)out + elem, 16), x, sizeof(x));
}

// What a query row sees of the drafted tokens' own rows.
struct PagedRow {
    int row_of;      // index into [B][nl][H_q][n] of row r
    int token;       // of the call, or -1: not a row of it
};
__device__ inline PagedRow paged_row(const PagedAttend &a, int hd, int r, int cnt)
{
    const int i = a.n == 1 ? 0 : r / a.G, j = r - i * a.G;
    return {(hd * a.G + j) * a.n + i, r < a.R && i < cnt ? i : -1};      // hd = (b * nl + l) * H + h
}

// The lowest n bits.
__device__ inline unsigned long long low_bits(int n)
{
    return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
}
// Which of the rows t0 .. t0 + 63 of sequence b token i sees; base: the first of the tokens' own rows, len: the rows there are.
__device__ inline unsigned long long sees(const PagedAttend &a, int b, int i, int t0, int base, int len)
{
    if (i < 0) return 0;
    if (!a.mask) return low_bits(min(base + i + 1, len) - t0);
    unsigned long long s = low_bits(base - t0);
    const int words = (a.n + 63) >> 6, j0 = t0 - base;       // bit j of the mask is row t0 + (j - j0)
    const unsigned long long *m = a.mask + ((size_t)b * a.n + i) * words;
    if (j0 >= 0) {
        const int w = j0 >> 6, sh = j0 & 63;
        if (w < words) s |= m[w] >> sh;
        if (sh && w + 1 < words) s |= m[w + 1] << (64 - sh);
    } else if (j0 > -64)
        s |= m[0] << -j0;
    return s & low_bits(len - t0);
}

// x where the bit of `word` is set, otherwise -inf; two vector instructions, and no scalar registers for conditions.
__device__ inline float seen_or_none(unsigned word, int bit, float x)
{
    const unsigned all = (unsigned)__builtin_amdgcn_sbfe((int)word, bit, 1);
    return __uint_as_float((all & __float_as_uint(x)) | (~all & 0xff800000u));
}

// Where the 16-row parts of a head's cache are: scalar code, whose loads of table entries do not count among those of the tiles.
struct PageWalk {
    const char *k, *v;                 // the head's rows of page 0
    const int32_t *table;              // the sequence's
    size_t stride;                     // bytes from a page to the next
    int pages, psh, last, row_bytes;   // last: the sequence's last row
    __device__ PageWalk(const PagedGeo &g, int b, int hd, int len, int row_bytes_)
        : table(g.table + (size_t)b * g.width), pages(g.pages), psh(g.psh), last(max(len - 1, 0)), row_bytes(row_bytes_)
    {
        const size_t head = ((size_t)(g.l0 * g.H + (hd - b * g.nl * g.H)) << g.psh) * row_bytes_;
        k = (const char *)g.k + head;
        v = (const char *)g.v + head;
        stride = ((size_t)g.L * g.H << g.psh) * row_bytes_;
    }
    // the page of row r, or of the last one where r is behind it; its entry may name none
    __device__ int entry(int r) const { return ((const __attribute__((address_space(4))) int32_t *)table)[min(r, last) >> psh]; }
    __device__ bool has(int id) const { return (unsigned)id < (unsigned)pages; }
    // bytes from k or v to row r of that page; of page 0 if there is none
    __device__ size_t offset(int id, int r) const
    {
        return (has(id) ? (unsigned)id : 0u) * stride + (unsigned)((r & ((1 << psh) - 1)) * row_bytes);
    }
};

// Eight weights as three matrix operands whose sum they are, exactly: 8 bits of the 24 each.
__device__ inline unsigned high_halves(float a, float b)
{
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ inline float top8(float x)
{
    return __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}
__device__ inline void weights_to_bf16(const float (&p)[8], bf16x8_t (&t)[3])
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        pu4_t u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = high_halves(x[2 * i], x[2 * i + 1]);
        t[k] = __builtin_bit_cast(bf16x8_t, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= top8(x[i]);
    }
}

// 16 rows of the lane's 16-lane group, four elements each, as columns: lane n gives the address of elements 4 (n % 4) .. + 4 of row
// n / 4 of four rows of 16, and gets element n of each of them.
__device__ inline pu2_t column_read(unsigned lds)
{
    return __builtin_bit_cast(pu2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) ps4_t *)(size_t)lds));
}

// Bits 15 and 31 set where the halves are bf16 numbers that are not finite; other bits may be set too.
__device__ inline unsigned not_finite(unsigned u)
{
    return (u & 0x7fff7fffu) + 0x00800080u;
}
__device__ inline unsigned not_finite(pu4_t u)
{
    return not_finite(u.x) | not_finite(u.y) | not_finite(u.z) | not_finite(u.w);
}
// Elements that are not finite, as ones; or the finite ones, the others zero.
__device__ inline pu4_t not_finite_or_rest(pu4_t u, bool ones)
{
    pu4_t y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned top = not_finite(u[e]) & 0x80008000u, all = (top - (top >> 15)) | top;
        y[e] = ones ? all & 0x3f803f80u : u[e] & ~all;
    }
    return y;
}

// Tiles in shared memory (of the token kernel TR rows, 8 KB, a wavefront's own).  16-byte unit u of row r stands at position u ^ swz(r) of
// the row: eight lanes that read one unit of eight rows meet distinct banks, and so do 32 that read two units of eight rows or four units
// of four as columns (with 2 (r % 8) for d = 128 the latter met two by two: a third of the shared memory's time for 512 tokens).
template <int DH>
struct PagedTile {
    static constexpr int UN = DH / 8, TR = 4096 / DH, SUB = TR / 16;   // units of a row, rows, 16-row parts
    static constexpr int ROW = DH * 2, PART = 16 * ROW;                // bytes
    static __device__ unsigned swz(unsigned r) { return (DH == 128 ? (r & 3) << 2 : (r & 2) << 1) | (r & 4) >> 1; }
};
template <int DH, int MT, int NW>
struct PagedTokenSmem {
    union {
        alignas(256) unsigned char tile[NW][2][8192];   // [wavefront][K, V]
        alignas(16) float o[NW][4096];                  // rows of d, in the wavefront's own tiles: others may still be reading theirs
    };
    float m[NW][16 * MT], l[NW][16 * MT];
    static_assert(sizeof(tile) == sizeof(o) && 16 * MT * DH <= 4096, "a wavefront's results lie in its tiles");
    // 16-byte unit u of row `row` of o, spread over the banks
    static __device__ int unit(int row, int u) { return row * DH + (u ^ (row & (DH / 4 - 1) & 15)) * 4; }
};

// Up to 32 query rows of a KV-head, one pass over the rows with the running maximum and sum of every query row.
//   S^T (16 keys x 16 rows) = K Q^T and O^T (16 dimensions x 16 rows) += V^T P^T by 16 x 16 x 32 products: a lane has four keys of ONE row
//   in each 16-row part, so that maximum and sum meet over four lanes at the end of a tile, and the elements of two parts are P^T's operand as they
//   stand; V^T's is read from the rows as columns, which the hardware does on the way out of shared memory.
// Bound by the bytes of the cache.  So every wavefront has tiles of its own (K and V of 4096 elements each), which go straight from
// global to shared memory and are asked for as soon as the products have read the tile before: no registers, no barrier between wavefronts, and
// 64 to 128 KB of every compute unit under way or in use all the time.  Weights are three bf16 terms, exactly, which the matrix unit has time for (9 % busy).
// One token, 30 layers of 8 KV-heads, 15512 rows: 1.907 GB in 278 us, 6.85 TB/s, what a loop of loads reaches (301 with tiles that
// wavefronts share).  8 KV-heads of one layer, 1064 rows: 11.4 us, a chain of five tiles for each of eight wavefronts.
// Tiles ta .. tb - 1 of block rb of head (b, hd)'s rows; slot: where a piece's result goes (-1: the block is whole).
template <int DH, int MT, bool NTL, int NW>
__device__ inline void paged_token_block(const PagedAttend &a, PagedTokenSmem<DH, MT, NW> &sm, const PartSeq &sq, int b, int hd, int rb,
                                         int ta, int tb, int slot)
{
    using T = PagedTile<DH>;
    constexpr int NS = DH / 32, ND = DH / 16, RB = 16 * MT, LOADS = 4096 * 2 / 1024;
    const PagedGeo &g = a.g;
    const int len = sq.len, cnt = min(sq.cnt, len), base = len - cnt;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const PageWalk pages(g, b, hd, len, T::ROW);

    // cache rows that the block's last and first row may see
    const int last = min(cnt - 1, min(rb * RB + RB - 1, a.R - 1) / a.G), first = rb * RB / a.G;
    const int seen = cnt <= first ? 0 : a.mask ? len : base + last + 1;
    const int full = (int)uniform(a.mask ? base : base + first + 1);
    const int t_end = (int)uniform(min(tb, (seen + T::TR - 1) / T::TR));
    int t = ta + wave;

    const unsigned lds_k = __builtin_amdgcn_readfirstlane(lds_address(sm.tile[wave][0])),
                   lds_v = __builtin_amdgcn_readfirstlane(lds_address(sm.tile[wave][1]));
    // lane i's 16 bytes of a load of 1 KB land at 16 i: which unit of which row that is
    unsigned off[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const unsigned r = j * (64 / T::UN) + lane / T::UN, u = lane % T::UN;
        off[j] = r * T::ROW + (u ^ T::swz(r)) * 16;
    }
    // The pages of a tile's 16-row parts, as bytes from the head's rows of page 0.
    struct Parts {
        size_t at[T::SUB];
        unsigned gone;       // bit s: part s has no page
    };
    auto parts_of = [&](int t) {
        Parts p;
        int id[T::SUB];
        p.gone = 0;
#pragma unroll
        for (int s = 0; s < T::SUB; ++s) id[s] = pages.entry(t * T::TR + s * 16);
#pragma unroll
        for (int s = 0; s < T::SUB; ++s) {
            p.gone |= pages.has(id[s]) ? 0u : 1u << s;
            p.at[s] = pages.offset(id[s], t * T::TR + s * 16);
        }
        return p;
    };
    auto load = [&](const char *pool, const Parts &p, unsigned lds) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            constexpr int PER = LOADS / T::SUB;       // loads of a part
            const char *from = pool + p.at[j / PER] + (j % PER & ~1) * 1024;
            const unsigned o = off[j % PER & 1];
            NTL ? stream_to_lds(from, o, lds + j * 1024) : load_to_lds(from, o, lds + j * 1024);
        }
    };
    Parts now, next;
    if (t < t_end) {
        now = parts_of(t);
        load(pages.k, now, lds_k);
        load(pages.v, now, lds_v);
        next = parts_of(min(t + NW, t_end - 1));
    }

    PagedRow qr[MT];
    bf16x8_t qf[MT][NS];
    float crow[MT], m[MT], sum[MT];
    pf4_t o[MT][ND];
#pragma unroll
    for (int r = 0; r < MT; ++r) {
        qr[r] = paged_row(a, hd, rb * RB + r * 16 + col, cnt);
        unsigned odd = 0;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            pu4_t u = {0, 0, 0, 0};
            if (qr[r].token >= 0) u = *(const pu4_t *)(a.q + (size_t)qr[r].row_of * DH + s * 32 + quarter * 8);
            odd |= not_finite(u);
            qf[r][s] = __builtin_bit_cast(bf16x8_t, u);
        }
        crow[r] = quarters_max(odd & 0x80008000u ? 1.f : 0.f) > 0.f ? __uint_as_float(0x7fc00000u) : a.scale;
        m[r] = -INFINITY;
        sum[r] = 0.f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[r][dt] = pf4_t{0.f, 0.f, 0.f, 0.f};
    }
    // K: row col of a part, unit 4 s + quarter; V: row 4 quarter + col / 4, two units of 16 elements dt, of which the lane reads 8 bytes
    const unsigned k_at = lds_k + col * T::ROW + (quarter ^ T::swz(col)) * 16;
    const unsigned v_row = quarter * 4 + col / 4, v_at = lds_v + v_row * T::ROW + T::swz(v_row) * 16 + (col & 3) * 8;

    for (; t < t_end; t += NW) {
        const bool masked = t * T::TR + T::TR > full || now.gone;   // some row does not see all of the tile
        const bool more = t + NW < t_end;
        const unsigned gone = now.gone;
        float x[MT][T::SUB][4];
        lds_loads_wait<LOADS>();       // K is there, V may be under way
#pragma unroll
        for (int kb = 0; kb < T::SUB; ++kb) {
            pf4_t c[MT] = {};
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const bf16x8_t k = frag_read((k_at ^ s * 64) + kb * T::PART);
#pragma unroll
                for (int r = 0; r < MT; ++r) c[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[r][s], c[r], 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[r][kb][i] = c[r][i] * crow[r];
        }
        __builtin_amdgcn_sched_barrier(0);
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the bytes have been read
        if (more) load(pages.k, next, lds_k);
        __builtin_amdgcn_sched_barrier(0);

        unsigned long long here = 0;       // rows of the tile that there are
        if (masked) {
            here = low_bits(len - t * T::TR);
#pragma unroll
            for (int s = 0; s < T::SUB; ++s)
                if (gone >> s & 1) here &= ~(0xffffull << (16 * s));
        }
        unsigned long long see[MT];
        bf16x8_t p[MT][T::SUB / 2][3];
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            if (masked) {
                see[r] = (sees(a, b, qr[r].token, t * T::TR, base, len) & here) >> (quarter * 4);
#pragma unroll
                for (int kb = 0; kb < T::SUB; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        x[r][kb][i] = seen_or_none((unsigned)(see[r] >> (kb / 2 * 32)), kb % 2 * 16 + i, x[r][kb][i]);
            }
            float mt = m[r];
#pragma unroll
            for (int kb = 0; kb < T::SUB; ++kb) mt = fmaxf(mt, fmaxf(fmaxf(x[r][kb][0], x[r][kb][1]), fmaxf(x[r][kb][2], x[r][kb][3])));
            mt = quarters_max(mt);
            if (__any(mt > m[r])) {
                const float alpha = exp2_hw(m[r] - finite_or_zero(mt));
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) o[r][dt] *= alpha;
                sum[r] *= alpha;
                m[r] = mt;
            }
            const float mz = finite_or_zero(m[r]);
#pragma unroll
            for (int kb = 0; kb < T::SUB; ++kb) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[r][kb][i] = exp2_hw(x[r][kb][i] - mz);
                sum[r] += (x[r][kb][0] + x[r][kb][1]) + (x[r][kb][2] + x[r][kb][3]);
            }
#pragma unroll
            for (int c = 0; c < T::SUB / 2; ++c) {
                const float w[8] = {x[r][2 * c][0],     x[r][2 * c][1],     x[r][2 * c][2],     x[r][2 * c][3],
                                    x[r][2 * c + 1][0], x[r][2 * c + 1][1], x[r][2 * c + 1][2], x[r][2 * c + 1][3]};
                weights_to_bf16(w, p[r][c]);
            }
        }
        if (more)
            lds_loads_wait<LOADS>();     // V is there, the next K may be under way
        else
            lds_loads_wait<0>();
        auto v_read = [&](int dt, int c) {
            const unsigned at = (v_at ^ dt * 32) + 2 * c * T::PART;
            const pu2_t y0 = column_read(at), y1 = column_read(at + T::PART);
            return pu4_t{y0.x, y0.y, y1.x, y1.y};
        };
        if (masked) {
            // Rows that are not there may hold anything: zeros instead.  An element that is not finite makes that of the output
            // NaN for the rows that see it, and is zero for the others: a weight of zero would not be enough.
            unsigned odd = 0;
#pragma unroll 1
            for (int j = 0; j < LOADS; ++j) {
                const unsigned at = lds_v + j * 1024 + lane * 16, r = (unsigned)(j * 64 + lane) / T::UN;
                pu4_t u = __builtin_bit_cast(pu4_t, frag_read(at));
                if (!(here >> r & 1)) {
                    u = pu4_t{0, 0, 0, 0};
                    *(__attribute__((address_space(3))) pu4_t *)(size_t)at = u;
                }
                odd |= not_finite(u);
            }
            __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if ((a.n > 1 || a.mask) && __any(odd & 0x80008000u)) {
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    bf16x8_t ones[T::SUB / 2];
#pragma unroll
                    for (int c = 0; c < T::SUB / 2; ++c) {
                        pu4_t u;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const unsigned two = (unsigned)(see[r] >> (32 * c + 16 * (i / 2) + 2 * (i % 2))) & 3u;
                            u[i] = (two & 1 ? 0x3f80u : 0u) | (two & 2 ? 0x3f800000u : 0u);
                        }
                        ones[c] = __builtin_bit_cast(bf16x8_t, u);
                    }
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) {
                        pf4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int c = 0; c < T::SUB / 2; ++c)
                            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, not_finite_or_rest(v_read(dt, c), true)),
                                                                        ones[c], y, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (y[i] > 0.f) o[r][dt][i] = __uint_as_float(0x7fc00000u);
                    }
                }
                __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
                for (int j = 0; j < LOADS; ++j) {
                    const unsigned at = lds_v + j * 1024 + lane * 16;
                    *(__attribute__((address_space(3))) pu4_t *)(size_t)at =
                        not_finite_or_rest(__builtin_bit_cast(pu4_t, frag_read(at)), false);
                }
                __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int c = 0; c < T::SUB / 2; ++c) {
                const bf16x8_t v = __builtin_bit_cast(bf16x8_t, v_read(dt, c));
#pragma unroll
                for (int r = 0; r < MT; ++r)
#pragma unroll
                    for (int k = 0; k < 3; ++k) o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[r][c][k], o[r][dt], 0, 0, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) {
            load(pages.v, next, lds_v);
            now = next;
            next = parts_of(min(t + 2 * NW, t_end - 1));
        }
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
        for (int dt = 0; dt < ND; ++dt) *(pf4_t *)&sm.o[wave][sm.unit(r * 16 + col, dt * 4 + quarter)] = o[r][dt];
    }
    __syncthreads();
    const PagedAttend &z = late_args<PagedAttend>();
    for (int row = threadIdx.x >> 4; row < RB; row += NW * 4) {
        const int d0 = (threadIdx.x & 15) * (DH / 16);
        const PagedRow rr = paged_row(z, hd, rb * RB + row, cnt);
        if (rr.token < 0) continue;
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
                const pf4_t y = *(const pf4_t *)&sm.o[w][sm.unit(row, (d0 + e) / 4)];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e + k] += f * y[k];
            }
        }
        if (slot >= 0) {
            const size_t at = (size_t)(z.group() * 2 + slot) * RB + row;
            __builtin_memcpy(__builtin_assume_aligned(z.ws_o + at * DH + d0, 16), x, sizeof(x));
            if (d0 == 0) z.ws_ml[at] = make_float2(mm, ll);
        } else {
            const float inv = 1.f / ll;
#pragma unroll
            for (int e = 0; e < DH / 16; ++e) x[e] = ll == 0.f ? 0.f : x[e] * inv;     // (where no row has weight, x may be NaN)
            store_out<DH / 16>(z.out, z.bf16, (size_t)rr.row_of * DH + d0, x);
            if (d0 == 0 && z.lse) z.lse[rr.row_of] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * P_LN2;
        }
    }
}

template <int DH, int MT, bool NTL, int NW>
__global__ __launch_bounds__(64 * NW, 2) void paged_token_kernel(PagedAttend a)
{
    __shared__ PagedTokenSmem<DH, MT, NW> sm;
    run_parts(a, [&](const PartSeq &sq, int b, int hd, int rb, int ta, int tb, int slot) {
        paged_token_block<DH, MT, NTL, NW>(a, sm, sq, b, hd, rb, ta, tb, slot);
    });
}

// Many query rows.  A work-group of NW wavefronts has blocks of RB = 256 (NW 8), 128 or 64 (4) rows, and all of its wavefronts use the same
// tiles of 64 cache rows, which go straight from global to one of two buffers in shared memory while the tile in the other is
// in use; of four wavefronts each loads a part of 16 rows of K and of V, of eight four do for K and four for V.
//   S^T (32 keys x 32 rows) = K Q^T and O^T (32 dimensions x 32 rows) += V^T P^T by 32 x 32 x 16 products (see wnw_lds.h for
//   operands): a lane has 16 keys of ONE row, elements 0 .. 7 in the 16-row part 2 k and 8 .. 15 in 2 k + 1, so that S^T's elements are P^T's
//   operand as they stand, and V^T's is read from the rows as columns.
// KS = 2, for 33 to 64 rows: two wavefronts share 32 rows, each with half of every tile's keys, and join at the end.
// A row's maximum m is raised, and its output and sum scaled, only when a logit exceeds it by LAZY_P (base 2).
// A weight is three bf16 terms, exactly, whatever the outputs' type.  As one term 13 to 31 % of bf16 outputs were not the fp32 ones rounded, which
// is what the flag promises and what up to 32 rows get (512 tokens below would take 280 us and not 446 to 468); as two, rounded to 17 bits, still
// 0.06 to 0.16 % were not nearest, where three leave the 0.02 to 0.06 % of fp32 sums (381 us).
// Bound by the matrix unit and, beside it, the vector unit and shared memory, in the card's power limit.  Hence 32 rows a wavefront, for each of which
// K's and V's operands are read once from shared memory; K is a round ahead, so that the next tile's products with K run
// between the vector instructions of this one's softmax; and 256 rows a work-group, which halve the bytes that are loaded per row.  512 tokens, 2 layers
// of 32 heads over 8, 15512 rows: 256 GFLOP, of which V's half is done three times, in 446 to 468 us, so 1100-1150 TFLOP/s of the matrix unit; an
// 8192^3 product reaches 1150-1230.  Measured with one term a weight: four buffers for K and V each were 5 to 10 % slower (addresses that differ
// between rounds), units moved once more in odd parts 2 % (no bank conflicts left, but registers in memory).
// MASKED tiles are the causal edge, a draft's own rows, missing pages and the end of a sequence.
constexpr float LAZY_P = 8.f;

template <int DH>
struct PagedWideSmem {
    alignas(256) unsigned char tile[2][2][64 * DH * 2];   // [K, V][buffer]
    unsigned dirty[2][4];      // a wavefront's part of V has a number that is not finite
};
// In the tiles' place at the end, where two wavefronts share 32 rows: sums, maximum and sum of weights of the second.
template <int DH>
struct PagedWideJoin {
    pf4_t o[2][DH / 8][64];
    float2 ml[2][64];
};

template <int DH, int KS, bool NTL, int NW>
__device__ inline void paged_wide_block(const PagedAttend &a, PagedWideSmem<DH> &sm, const PartSeq &sq, int b, int hd, int rb, int ta,
                                        int tb, int slot)
{
    using T = PagedTile<DH>;
    constexpr int NS = DH / 16, ND = DH / 32, RB = 32 * NW / KS, NB = 2 / KS, PL = 16 * T::ROW / 1024;   // PL: loads of a part
    constexpr unsigned BUF = 64 * DH * 2, V_OFF = 2 * BUF;
    const PagedGeo &g = a.g;
    const int len = sq.len, cnt = min(sq.cnt, len), base = len - cnt;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int rows32 = KS == 2 ? wave & 1 : wave, key32 = KS == 2 ? wave >> 1 : 0;    // the wavefront's rows, and its keys of a tile
    const PageWalk pages(g, b, hd, len, T::ROW);

    // cache rows that the block's last and first row may see
    const int last = min(cnt - 1, min(rb * RB + RB - 1, a.R - 1) / a.G), first = rb * RB / a.G;
    const int seen = cnt <= first ? 0 : a.mask ? len : base + last + 1;
    const int full = (int)uniform(a.mask ? base : base + first + 1);
    const int t_end = (int)uniform(min(tb, (seen + 63) / 64));

    const unsigned lds = uniform(lds_address(sm.tile[0][0]));
    unsigned off[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const unsigned r = j * (64 / T::UN) + lane / T::UN, u = lane % T::UN;
        off[j] = r * T::ROW + (u ^ T::swz(r)) * 16;
    }
    // the wavefront's part of a tile, as bytes from the head's rows of page 0, and which of the four parts have no page
    struct Parts {
        size_t at;
        unsigned gone;
    };
    auto parts_of = [&](int t) {
        int id[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) id[s] = pages.entry(t * 64 + s * 16);
        Parts p = {pages.offset(wave & 2 ? (wave & 1 ? id[3] : id[2]) : (wave & 1 ? id[1] : id[0]), t * 64 + (wave & 3) * 16), 0};
#pragma unroll
        for (int s = 0; s < 4; ++s) p.gone |= pages.has(id[s]) ? 0u : 1u << s;
        return p;
    };
    // of four wavefronts each loads a part of K and of V, of eight four do for K and four for V
    const int part = wave & 3;
    const bool has_k = NW == 4 || wave < 4, has_v = NW == 4 || wave >= 4;
    auto load = [&](const char *pool, const Parts &p, unsigned to) {
#pragma unroll
        for (int j = 0; j < PL; ++j) {
            const char *from = pool + p.at + (j & ~1) * 1024;
            const unsigned at = lds + to + part * T::PART + j * 1024;
            NTL ? stream_to_lds(from, off[j & 1], at) : load_to_lds(from, off[j & 1], at);
        }
    };
    // K of a tile is there a round before its V: buffers of K 0, 1, then of V
    Parts now = {0, 0}, next = {0, 0}, after = {0, 0};
    if (ta < t_end) {
        now = parts_of(ta);
        next = parts_of(ta + 1);
        after = parts_of(ta + 2);
        if (has_k) {
            load(pages.k, now, 0);
            load(pages.k, next, BUF);
        }
        if (has_v) load(pages.v, now, V_OFF);
    }

    const PagedRow qr = paged_row(a, hd, rb * RB + rows32 * 32 + col, cnt);
    bf16x8_t qf[NS];
    unsigned odd = 0;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        pu4_t u = {0, 0, 0, 0};
        if (qr.token >= 0) u = *(const pu4_t *)(a.q + (size_t)qr.row_of * DH + s * 16 + half * 8);
        odd |= not_finite(u);
        qf[s] = __builtin_bit_cast(bf16x8_t, u);
    }
    odd |= (unsigned)__shfl_xor((int)odd, 32);
    const float crow = odd & 0x80008000u ? __uint_as_float(0x7fc00000u) : a.scale;
    float m = -INFINITY, sum = 0.f;
    f32x16_t o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    // K: row col, unit 2 s + half; V: rows 4 half + col16 / 4 and 8 more, two units of dimensions 16 (lane / 16 % 2) .. + 16
    const unsigned k_get = lds + (key32 * 32 + col) * T::ROW + (half ^ T::swz(col)) * 16;
    const unsigned n16 = lane & 15, v_row = half * 4 + n16 / 4;
    const unsigned v_get = lds + V_OFF + (key32 * 32 + v_row) * T::ROW + ((2 * (lane >> 4 & 1)) ^ T::swz(v_row)) * 16 + (n16 & 3) * 8;

    auto logits = [&](f32x16_t (&x)[NB], unsigned buf) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                const f32x16_t zero = {};
                x[kb] = mfma32(frag_read((k_get ^ s * 32) + kb * 32 * T::ROW + buf), qf[s], s ? x[kb] : zero);
            }
    };
    f32x16_t x[NB];      // products of the tile that is next
    if (ta < t_end) {
        lds_loads_wait<0>();
        lds_tile_barrier();
        logits(x, 0);
    }
    // one tile, whose K and V are in the buffers at `buf`: its softmax beside the next one's products with K, then its products with V.
    // MASKED: some row may not see all of the tile.
    auto round = [&](int t, auto buf_c, auto masked_c) {
        const unsigned buf = buf_c, other = BUF - buf;
        constexpr bool MASKED = decltype(masked_c)::value;
        const int side = buf ? 1 : 0;
        unsigned long long here = ~0ull;       // rows of the tile that there are
        lds_loads_wait<0>();
        if constexpr (MASKED) {
            here = low_bits(len - t * 64);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (now.gone >> s & 1) here &= ~(0xffffull << (16 * s));
            // Rows that are not there may hold anything: zeros instead.
            unsigned odd = 0;
#pragma unroll 1
            for (int j = has_v ? 0 : PL; j < PL; ++j) {
                const unsigned at = lds + buf + V_OFF + part * T::PART + j * 1024 + lane * 16, r = part * 16 + (unsigned)(j * 64 + lane) / T::UN;
                pu4_t u = __builtin_bit_cast(pu4_t, frag_read(at));
                if (!(here >> r & 1)) {
                    u = pu4_t{0, 0, 0, 0};
                    *(__attribute__((address_space(3))) pu4_t *)(size_t)at = u;
                }
                odd |= not_finite(u);
            }
            const bool any = __any(odd & 0x80008000u);
            if (has_v && lane == 0) sm.dirty[side][part] = any;
        }
        lds_tile_barrier();
        if (has_k && t + 2 < t_end) load(pages.k, after, buf);
        if (has_v && t + 1 < t_end) load(pages.v, next, V_OFF + other);
        // element i of x[kb] is of the wavefront's key 32 kb + 8 (i / 4) + 4 half + i % 4; base-2 logits relative to m from here
        float mz = finite_or_zero(m);
        f32x16_t y[NB];
        if constexpr (!MASKED) {
            __builtin_amdgcn_sched_barrier(0);
            logits(y, other);
        }
        float w[2 * NB][8];        // of 16-row part c: elements 8 (c % 2) .. + 8 of x[c / 2]
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) w[c][i] = fmaf(x[c >> 1][8 * (c & 1) + i], crow, -mz);
        unsigned long long see = ~0ull;
        if constexpr (MASKED) {
            see = (sees(a, b, qr.token, t * 64, base, len) & here) >> (key32 * 32 + half * 4);
#pragma unroll
            for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[c][i] = seen_or_none((unsigned)(see >> (c & 2 ? 32 : 0)), 16 * (c & 1) + 8 * (i / 4) + i % 4, w[c][i]);
        }
        float top = w[0][0];
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, w[c][i]);
        {
            auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
        }
        if constexpr (!MASKED) {
            // a read of K, a product and its share of the vector instructions in turn
#pragma unroll
            for (int i = 0; i < 3; ++i) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
            for (int i = 0; i < NS * NB; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            }
        }
        const bool up = top > (m == -INFINITY ? -INFINITY : LAZY_P);
        if (__any(up)) {      // (a row's own logits decide, so that its results do not depend on the rows beside it)
            const float mn = up ? mz + top : m, rise = finite_or_zero(mn) - mz, alpha = m == -INFINITY ? 0.f : exp2_hw(-rise);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= alpha;
#pragma unroll
            for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[c][i] -= rise;
            sum *= alpha;
            m = mn;
        }
        bf16x8_t p[2 * NB][3];
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[c][i] = exp2_hw(w[c][i]);
            sum += ((w[c][0] + w[c][1]) + (w[c][2] + w[c][3])) + ((w[c][4] + w[c][5]) + (w[c][6] + w[c][7]));
            weights_to_bf16(w[c], p[c]);
        }
        auto v_read = [&](int dt, int c) {
            const unsigned at = (v_get ^ dt * 64) + c * T::PART + buf;
            const pu2_t y0 = column_read(at), y1 = column_read(at + 8 * T::ROW);
            return pu4_t{y0.x, y0.y, y1.x, y1.y};
        };
        if constexpr (MASKED)
            if (sm.dirty[side][0] | sm.dirty[side][1] | sm.dirty[side][2] | sm.dirty[side][3]) {
                // an element that is not finite makes that of the output NaN for the rows that see it, and is zero for the others
                pu4_t ones[2 * NB];
#pragma unroll
                for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned two = (unsigned)(see >> (16 * c + 8 * (i / 2) + 2 * (i % 2))) & 3u;
                        ones[c][i] = (two & 1) * 0x3f80u | (two >> 1) * 0x3f800000u;
                    }
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    f32x16_t found;
#pragma unroll
                    for (int c = 0; c < 2 * NB; ++c) {
                        const f32x16_t zero = {};
                        found = mfma32(__builtin_bit_cast(bf16x8_t, not_finite_or_rest(v_read(dt, c), true)), __builtin_bit_cast(bf16x8_t, ones[c]),
                                       c ? found : zero);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[dt][i] = found[i] > 0.f ? __uint_as_float(0x7fc00000u) : o[dt][i];
                }
                lds_tile_barrier();
#pragma unroll 1
                for (int j = has_v ? 0 : PL; j < PL; ++j) {
                    const unsigned at = lds + buf + V_OFF + part * T::PART + j * 1024 + lane * 16;
                    *(__attribute__((address_space(3))) pu4_t *)(size_t)at = not_finite_or_rest(__builtin_bit_cast(pu4_t, frag_read(at)), false);
                }
                lds_tile_barrier();
            }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int c = 0; c < 2 * NB; ++c) {
                const bf16x8_t v = __builtin_bit_cast(bf16x8_t, v_read(dt, c));
#pragma unroll
                for (int k = 0; k < 3; ++k) o[dt] = mfma32(v, p[c][k], o[dt]);
            }
        now = next;
        next = after;
        after = parts_of(t + 3);
        if constexpr (MASKED)
            logits(x, other);       // (here, as registers are short before)
        else
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) x[kb] = y[kb];
    };
    // tiles that every row sees, in pairs; then the others (all of them from the first page on that is not there)
    int t = ta;
    for (const int t_full = min(t_end, full / 64); t + 2 <= t_full && !(now.gone | next.gone); t += 2) {
        round(t, std::integral_constant<unsigned, 0>{}, std::false_type{});
        round(t + 1, std::integral_constant<unsigned, BUF>{}, std::false_type{});
    }
#pragma unroll 1
    for (; t < t_end; ++t) round(t, (t - ta) & 1 ? BUF : 0u, std::true_type{});
    sum += __shfl_xor(sum, 32);
    if constexpr (KS == 2) {
        // the keys' halves meet: the second's result to the same lane of the first's wavefront
        static_assert(sizeof(PagedWideJoin<DH>) <= sizeof(sm.tile));
        PagedWideJoin<DH> &jn = *(PagedWideJoin<DH> *)&sm;
        __syncthreads();
        if (key32) {
#pragma unroll
            for (int u = 0; u < ND * 4; ++u)
                jn.o[rows32][u][lane] = pf4_t{o[u / 4][u % 4 * 4], o[u / 4][u % 4 * 4 + 1], o[u / 4][u % 4 * 4 + 2], o[u / 4][u % 4 * 4 + 3]};
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
            const pf4_t y = jn.o[rows32][u][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[u / 4][u % 4 * 4 + e] = f0 * o[u / 4][u % 4 * 4 + e] + f1 * y[e];
        }
    }
    const bool live = qr.token >= 0;
    // element i of o[dt]: dimension 32 dt + 8 (i / 4) + 4 half + i % 4 of row col
    const bool none = slot < 0 && sum == 0.f;        // no row has weight, and o may be NaN
    const float inv = slot >= 0 ? 1.f : 1.f / sum;
    const size_t at = slot >= 0 ? (size_t)(a.group() * 2 + slot) * RB + rows32 * 32 + col : (size_t)qr.row_of;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = none ? 0.f : o[dt][i + e] * inv;
            const size_t to = at * DH + dt * 32 + 2 * i;
            if (slot < 0 && a.bf16) {
                // the halves' four dimensions of eight meet, so that a lane has all of eight
                unsigned u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = to_bf16(y[2 * e]) | (unsigned)to_bf16(y[2 * e + 1]) << 16;
                const auto p = __builtin_amdgcn_permlane32_swap(u[0], u[2], false, false), q = __builtin_amdgcn_permlane32_swap(u[1], u[3], false, false);
                if (live) *(pu4_t *)((uint16_t *)a.out + to + 8 * half) = pu4_t{p[0], q[0], p[1], q[1]};
            } else if (live) {
                float *f = (slot < 0 ? (float *)a.out : a.ws_o) + to + 4 * half;
                *(pf4_t *)f = pf4_t{y[0], y[1], y[2], y[3]};
                *(pf4_t *)(f + 8) = pf4_t{y[4], y[5], y[6], y[7]};
            }
        }
    if (!live) return;
    if (half == 0) {
        if (slot >= 0)
            a.ws_ml[at] = make_float2(m, sum);
        else if (a.lse)
            a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * P_LN2;
    }
}

template <int DH, int KS, bool NTL, int NW>
__global__ __launch_bounds__(64 * NW, 2) void paged_wide_kernel(PagedAttend a)
{
    __shared__ PagedWideSmem<DH> sm;
    run_parts(a, [&](const PartSeq &sq, int b, int hd, int rb, int ta, int tb, int slot) {
        paged_wide_block<DH, KS, NTL, NW>(a, sm, sq, b, hd, rb, ta, tb, slot);
    });
}

// Joins the pieces of a cache: sixteen threads have a row's pieces p, p + GP, ..., and a work-group 16 / GP rows of a head.  Every block's
// pieces are found again from the lengths as the first kernel did, so that there is no list and no atomic operation, and the order of the
// sum is fixed.  Bound by the pieces' bytes, which are still in the last-level cache: 65536 rows of about two pieces (4 sequences, 64 tokens, 8 layers
// of 32 heads) 13-16 us, a few rows of many pieces 5.
template <int DH, int GP>
__global__ __launch_bounds__(P_THREADS) void paged_join_kernel(PagedAttend a)
{
    constexpr int E = DH / 16, ROWS = 16 / GP;
    __shared__ float so[GP > 1 ? GP : 1][ROWS][DH];
    __shared__ float2 sml[GP > 1 ? GP : 1][ROWS];
    const unsigned groups = (a.R + ROWS - 1) / ROWS, hd = blockIdx.x / groups, r0 = (blockIdx.x - hd * groups) * ROWS;
    const int b = hd / (a.g.nl * a.g.H);
    const PartSeq sq = part_seq(a, b);
    const int cnt = min(sq.cnt, sq.len);
    if ((int)r0 >= cnt * a.G) return;
    PartShare<PagedAttend> sh;
    sh.init(a, threadIdx.x & 63);
    const PartPieces<PagedAttend> pc(a, sh, sq, b, hd, r0 >> a.rsh);
    if (pc.n == 1) return;
    const unsigned slot = threadIdx.x >> 4, rr = slot % ROWS, gp = slot / ROWS, r = r0 + rr, d0 = (threadIdx.x & 15) * E;
    const PagedRow row = paged_row(a, hd, r, cnt);
    float m = -INFINITY, sum = 0.f, x[E] = {};
    if (row.token >= 0) {
#pragma unroll 4
        for (unsigned p = gp; p < pc.n; p += GP) m = fmaxf(m, a.ws_ml[pc.at(p, r)].x);
        const float mz = finite_or_zero(m);
#pragma unroll 4
        for (unsigned p = gp; p < pc.n; p += GP) {
            const float2 ml = a.ws_ml[pc.at(p, r)];
            const float f = ml.y == 0.f ? 0.f : exp2f(ml.x - mz);       // 0: the piece saw nothing
            sum += f * ml.y;
            float o[E];
            __builtin_memcpy(o, __builtin_assume_aligned(a.ws_o + pc.at(p, r) * DH + d0, 16), sizeof(o));
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] += f * o[e];
        }
    }
    if constexpr (GP > 1) {
        if (d0 == 0) sml[gp][rr] = make_float2(m, sum);
#pragma unroll
        for (int e = 0; e < E; ++e) so[gp][rr][d0 + e] = x[e];
        __syncthreads();
        if (gp) return;
#pragma unroll
        for (int k = 0; k < GP; ++k) m = fmaxf(m, sml[k][rr].x);
        const float mz = finite_or_zero(m);
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
#pragma unroll
        for (int k = 0; k < GP; ++k) {
            const float2 ml = sml[k][rr];
            const float f = ml.y == 0.f ? 0.f : exp2f(ml.x - mz);
            sum += f * ml.y;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] += f * so[k][rr][d0 + e];
        }
    }
    if (row.token < 0) return;
    const float inv = 1.f / sum;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = sum == 0.f ? 0.f : x[e] * inv;     // (where no row has weight, x may be NaN)
    store_out<E>(a.out, a.bf16, (size_t)row.row_of * DH + d0, x);
    if (a.lse && d0 == 0) a.lse[row.row_of] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * P_LN2;
}

// ---- host ------------------------------------------------------------------------------------

thread_local char p_msg[256] = "no error";

wnw_status paged_fail(wnw_status st, const char *msg)
{
    strncpy(p_msg, msg, sizeof p_msg - 1);
    return st;
}
wnw_status paged_hip()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WNW_OK : paged_fail(WNW_ERR_HIP, hipGetErrorString(e));
}
bool off16(const void *p)
{
    return (uintptr_t)p & 15;
}
bool off4(const void *p)
{
    return (uintptr_t)p & 3;
}

wnw_status paged_config(const wnw_paged_config *c, int32_t first_layer, int32_t n_layers, int32_t n)
{
    if (!c) return paged_fail(WNW_ERR_INVALID, "NULL configuration");
    if (c->batch < 1 || c->layers < 1 || c->kv_heads < 1 || c->pages < 1 || c->table_width < 1)
        return paged_fail(WNW_ERR_INVALID, "batch, layers, kv_heads, pages and table_width must be at least 1");
    if (c->head_dim != 64 && c->head_dim != 128) return paged_fail(WNW_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256)
        return paged_fail(WNW_ERR_UNSUPPORTED, "page must be 16, 32, 64, 128 or 256");
    if (c->table_width > P_MAX_CAP / c->page) return paged_fail(WNW_ERR_UNSUPPORTED, "capacity above 2^24 rows");
    if (c->flags & ~(uint32_t)WNW_F_OUT_BF16) return paged_fail(WNW_ERR_INVALID, "unknown flag bits");
    if (first_layer < 0 || n_layers < 1 || first_layer > c->layers - n_layers)
        return paged_fail(WNW_ERR_INVALID, "layers outside the cache's");
    if (n < 0 || n > c->table_width * c->page) return paged_fail(WNW_ERR_INVALID, "n outside 0 .. capacity");
    if ((int64_t)c->batch * n_layers > INT32_MAX / 2 / c->kv_heads) return paged_fail(WNW_ERR_UNSUPPORTED, "too many heads");
    if ((int64_t)c->pages * c->layers > INT64_MAX / (256 * 128 * 2) / c->kv_heads) return paged_fail(WNW_ERR_UNSUPPORTED, "too many pages");
    return WNW_OK;
}
wnw_status paged_cache(const wnw_paged_cache *c)
{
    if (!c || !c->k || !c->v || !c->table) return paged_fail(WNW_ERR_INVALID, "NULL cache pointer");
    if (off16(c->k) || off16(c->v)) return paged_fail(WNW_ERR_INVALID, "pages must be aligned to 16 bytes");
    if (off4(c->table)) return paged_fail(WNW_ERR_INVALID, "the table must be aligned to 4 bytes");
    return WNW_OK;
}
PagedGeo paged_geo(const wnw_paged_config &c, const wnw_paged_cache &k, int32_t l0, int32_t nl)
{
    return PagedGeo{c.batch, c.layers, c.kv_heads, l0, nl, c.pages, c.table_width, __builtin_ctz((unsigned)c.page),
                    (uint16_t *)k.k, (uint16_t *)k.v, k.table};
}

template <typename F>
void paged_dispatch(const wnw_paged_config &c, F f)
{
    c.head_dim == 64 ? f(std::integral_constant<int, 64>{}) : f(std::integral_constant<int, 128>{});
}

// Times in us that decide how work is shared, measured on even batches: a whole block's start; a tile of a block that has a compute
// unit to itself (`own`), and of one when the chip is full, as a compute unit's time (`full`); what shares cost a call beside their tiles
// (the search, the parts' results, the join and its launch).
struct PagedPrice {
    double start, own, full, join;
};
PagedPrice paged_price(int RB, int head_dim, bool stream)
{
    const bool d64 = head_dim == 64;
    if (RB == 256) return d64 ? PagedPrice{9, 1.83, 2.03, 27} : PagedPrice{16, 2.83, 3.35, 42};
    if (RB == 128) return d64 ? PagedPrice{8, 1.36, 1.05, 18} : PagedPrice{14, 2.5, 2.05, 36};
    if (RB == 64) return d64 ? PagedPrice{7, 0.72, 0.85, 13} : PagedPrice{12, 1.1, 1.50, 18};
    if (RB == 32) return d64 ? PagedPrice{6, stream ? 0.38 : 0.25, 0.66, 11} : PagedPrice{7, stream ? 0.35 : 0.25, 0.68, 14};
    return d64 ? PagedPrice{5.5, stream ? 0.37 : 0.19, 0.62, 9} : PagedPrice{5, stream ? 0.34 : 0.165, 0.607, 11};
}

// Whether every block of rows gets a work-group of its own rather than the batch's tiles being cut into even parts that a second launch
// joins.  Measured whole and cut, a block's rows of the cache and what they took: one token, d = 128: 8 blocks of 1064 11.5 and
// 11.4, of 4000 25.5 and 13.2; 72 of 4000 29.2 and 30.6, of 15512 154 and 92; 128 of 1064 16 and 22, of 15512 174 and 157; 240 of 15512
// 276 and 294; d = 64: 72 of 1064 9.3 and 12.8, of 15512 81 and 50; 240 of 15512 141 and 152; five tokens of four heads: 8 of 1064 16.8
// and 15, 72 of 4000 44 and 38, 240 of 15512 299 and 341; blocks of 64 rows: 64 of 2000 48 and 40, 240 of 15512 358 and 354; of 128: 128 of 600 38
// and 47, of 2000 94 and 70, 256 of 2000 109 and 116, 240 of 15512 725 and 553; of 256: 64 of 600 44 and 46, of 2000 105 and 65, 128 of 2000 108 and
// 99, of 8000 366 and 274, 256 of 8000 491 and 518; d = 64: blocks of 128 rows, 128 of 600 21 and 28, of 2000 50 and 41, of 256 rows, 128 of
// 2000 69 and 61, 256 of 8000 288 and 307.
// Of a batch only the longest length is known here.  Whole blocks wait for the longest sequence's, which parts share out among all, so
// parts of several sequences are priced as if half of the rows were there.
// skew: the tokens' part of the rows, of which the first tokens see none (a prompt's blocks of 256 rows whole and cut: 128 of 1024 58 and 66,
// 126 of 2000 102 and 83, 122 of 7756 353 and 207, 256 of 2000 107 and 134, 504 of 4000 245 and 395, 486 of 7756 436 and 708, 976 of 7756 850 and 1373).
bool paged_whole(const PagedPrice &c, int RB, int64_t blocks, int64_t tiles, int batch, double skew)
{
    const double b = blocks / 256.0, t = (double)tiles;
    // (of the wide kernels' work-groups a compute unit holds one of 256 rows, two of others)
    const int64_t held = RB == 256 ? 256 : 512;
    const double turns = (held / 256) * std::min((double)((blocks + held - 1) / held), (double)blocks / held * (1 - skew / 2) + (1 - skew) / 2);
    const double later = RB == 256 ? c.start * std::max(0.0, b - 1) : 0.0;       // starts after the first
    const double whole = c.start + later + t * std::max(c.own, RB > 32 && b > 1 ? c.full * turns : c.full * b);
    const double cut = c.join + later + std::max(c.own * MIN_PIECE, c.full * t * b * (batch > 1 ? 0.5 : 1.0));
    return whole <= cut;
}

// How an attention call runs.
struct PagedPlan {
    int RB, W, tsh;     // RB 16, 32, 64, 128 or 256
    bool whole, eight, stream, join_groups;
    int64_t rows, o_bytes, ml_bytes;
    int64_t total() const { return o_bytes + ml_bytes; }
};
PagedPlan paged_plan(const wnw_paged_config &c, int32_t n_layers, int32_t q_heads, int32_t n, int32_t max_len)
{
    const int64_t cap = (int64_t)c.table_width * c.page, heads = (int64_t)c.batch * n_layers * c.kv_heads, R = (int64_t)q_heads / c.kv_heads * n;
    const int64_t len = max_len ? std::min<int64_t>(max_len, cap) : cap;
    PagedPlan p;
    p.RB = R > 128 ? 256 : R > 64 ? 128 : R > 32 ? 64 : R > 16 ? 32 : 16;
    p.tsh = c.head_dim == 64 || p.RB > 32 ? 6 : 5;
    const int64_t blocks = heads * ((R + p.RB - 1) / p.RB), per = (len + (1 << p.tsh) - 1) >> p.tsh, tiles = per * blocks;
    // bytes that one pass reads once and the 256 MB of the last-level cache cannot keep for the next one go past the caches (30 layers of 8
    // KV-heads, 15512 rows: 64 query rows of a KV-head 366 -> 348 us, 128 568 -> 554; rows that several blocks read must not:
    // 512 tokens 445 -> 474)
    p.stream = R <= p.RB && heads * len * c.head_dim * 4 > (256ll << 20);
    p.whole = paged_whole(paged_price(p.RB, c.head_dim, p.stream), p.RB, blocks, per, c.batch, R > p.RB ? std::min(1.0, n / (double)len) : 0.0);
    // Eight wavefronts instead of four for whole blocks that have a compute unit each (one token, 72 blocks of 4000 rows 41 -> 29 us; two blocks
    // of 16 rows take turns on the vector unit, so that 240 of 15512 rows take 299 with four and 316 with eight).
    p.eight = p.whole && p.RB <= 32 && blocks <= (p.RB == 16 ? 256 : 128) && len > 256;
    p.W = (int)std::max<int64_t>(1, p.whole ? blocks : std::min<int64_t>(p.RB == 256 ? 256 : 512, tiles / MIN_PIECE + blocks));
    p.rows = heads * R;
    // sixteen threads for each of a few rows' pieces, a thread group a row where there are many
    p.join_groups = p.rows <= 8192;
    p.o_bytes = p.whole ? 0 : (int64_t)p.W * 2 * p.RB * c.head_dim * 4;
    p.ml_bytes = p.whole ? 0 : (int64_t)p.W * 2 * p.RB * 8;
    return p;
}

template <int DH, int MT>
void launch_tokens(const PagedPlan &p, const PagedAttend &a, hipStream_t st)
{
    auto *k = p.eight ? (p.stream ? paged_token_kernel<DH, MT, true, 8> : paged_token_kernel<DH, MT, false, 8>)
                      : (p.stream ? paged_token_kernel<DH, MT, true, 4> : paged_token_kernel<DH, MT, false, 4>);
    hipLaunchKernelGGL(k, dim3(p.W), dim3(p.eight ? 512 : 256), 0, st, a);
}

template <int DH, bool NTL>
void launch_wide_as(const PagedPlan &p, const PagedAttend &a, hipStream_t st)
{
    auto *k = p.RB == 256 ? paged_wide_kernel<DH, 1, NTL, 8> : p.RB == 128 ? paged_wide_kernel<DH, 1, NTL, 4> : paged_wide_kernel<DH, 2, NTL, 4>;
    hipLaunchKernelGGL(k, dim3(p.W), dim3(p.RB == 256 ? 512 : 256), 0, st, a);
}

template <int DH>
void launch_wide(const PagedPlan &p, const PagedAttend &a, hipStream_t st)
{
    p.stream ? launch_wide_as<DH, true>(p, a, st) : launch_wide_as<DH, false>(p, a, st);
}

wnw_status paged_heads(const wnw_paged_config &c, int32_t n_layers, int32_t q_heads, int32_t n, int32_t max_len)
{
    if (q_heads < c.kv_heads || q_heads % c.kv_heads) return paged_fail(WNW_ERR_INVALID, "q_heads must be a multiple of kv_heads");
    if (max_len < 0) return paged_fail(WNW_ERR_INVALID, "negative max_len");
    if ((int64_t)c.batch * n_layers * q_heads > INT32_MAX / std::max(n, 1)) return paged_fail(WNW_ERR_UNSUPPORTED, "too many query rows");
    // the line of tiles is counted in 32 bits
    const int64_t blocks = ((int64_t)q_heads / c.kv_heads * n + 15) / 16 * c.batch * n_layers * c.kv_heads;
    const int64_t tiles = ((int64_t)c.table_width * c.page + 31) / 32;
    if (blocks > P_MAX_GROUPS || blocks > INT32_MAX / tiles) return paged_fail(WNW_ERR_UNSUPPORTED, "too many tiles for one call");
    return WNW_OK;
}

}  // namespace

}  // namespace wnw

using namespace wnw;

extern "C" {

const char *wnw_paged_last_error(void)
{
    return p_msg;
}

wnw_status wnw_rotary_frequencies(int32_t dim, double base, double factor, double low, double high, int64_t original_len, float *freq)
{
    if (dim < 0 || dim % 2) return paged_fail(WNW_ERR_INVALID, "dim must be even");
    if (!(base > 0.0) || !(factor >= 1.0) || std::isinf(base) || std::isinf(factor) || !(low >= 0.0) || !(high >= low) || original_len < 0)
        return paged_fail(WNW_ERR_INVALID, "base > 0, factor >= 1, 0 <= low <= high and original_len >= 0 are wanted");
    if (dim && !freq) return paged_fail(WNW_ERR_INVALID, "NULL pointer");
    for (int32_t i = 0; i < dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / dim), turns = (double)original_len * f / 6.283185307179586;
        // (low = high = infinity: every pair turns seldom)
        const double keep = turns < low ? 0.0 : turns > high ? 1.0 : high > low ? (turns - low) / (high - low) : 1.0;
        freq[i] = (float)(f * keep + f / factor * (1.0 - keep));
    }
    return WNW_OK;
}

wnw_status wnw_paged_append(const wnw_paged_config *cfg, const wnw_paged_cache *cache, const wnw_rotary *rotary, int32_t first_layer,
                            int32_t n_layers, int32_t q_heads, int32_t n, const void *k_dev, const void *v_dev, const void *q_dev,
                            void *q_out, const int32_t *at_dev, const int32_t *count_dev, const int32_t *position_dev, void *hip_stream)
{
    wnw_status st = paged_config(cfg, first_layer, n_layers, n);
    if (st == WNW_OK) st = paged_cache(cache);
    if (st != WNW_OK) return st;
    if (rotary) {
        if (rotary->dim < 0 || rotary->dim % 2 || rotary->dim > cfg->head_dim) return paged_fail(WNW_ERR_INVALID, "rotary: dim must be even, 0 .. head_dim");
        if (rotary->layout != WNW_ROTARY_HALVES && rotary->layout != WNW_ROTARY_PAIRS) return paged_fail(WNW_ERR_INVALID, "rotary: unknown layout");
        if (!std::isfinite(rotary->amplitude)) return paged_fail(WNW_ERR_INVALID, "rotary: the amplitude is not finite");
        if (rotary->dim && (!rotary->freq || off4(rotary->freq))) return paged_fail(WNW_ERR_INVALID, "rotary: NULL or misaligned frequencies");
    }
    if (n == 0) return WNW_OK;
    if (!k_dev != !v_dev || !q_dev != !q_out) return paged_fail(WNW_ERR_INVALID, "keys and values, and queries and their place, come together");
    if (cfg->kv_heads > (1 << 20)) return paged_fail(WNW_ERR_UNSUPPORTED, "more than 2^20 KV-heads");
    if (!k_dev && !q_dev) return paged_fail(WNW_ERR_INVALID, "NULL pointer");
    if (q_dev && (q_heads < 1 || q_heads > (1 << 20))) return paged_fail(WNW_ERR_INVALID, "q_heads must be 1 .. 2^20");
    if (!at_dev) return paged_fail(WNW_ERR_INVALID, "NULL pointer");
    if (off16(k_dev) || off16(v_dev) || off16(q_dev) || off16(q_out)) return paged_fail(WNW_ERR_INVALID, "rows must be aligned to 16 bytes");
    if (off4(at_dev) || off4(count_dev) || off4(position_dev)) return paged_fail(WNW_ERR_INVALID, "a pointer is not aligned to its elements");
    const int Hq = q_dev ? q_heads : 0, vectors = (k_dev ? 2 * cfg->kv_heads : 0) + Hq;
    const int dim = rotary ? rotary->dim : 0;
    int TT = 1;
    const int slots = P_THREADS / (cfg->head_dim / 8);
    while (TT < slots && TT < n) TT *= 2;
    const int64_t tiles = (n + TT - 1) / TT, layers = (int64_t)cfg->batch * n_layers;
    if (tiles * layers > P_MAX_GROUPS) return paged_fail(WNW_ERR_UNSUPPORTED, "too many rows for one call");
    // few work-groups: share a layer's vectors out to several
    const int rounds = (vectors + slots / TT - 1) / (slots / TT);
    const int64_t split = std::max<int64_t>(1, std::min<int64_t>(rounds, 2048 / (tiles * layers)));
    const PagedAppend a = {paged_geo(*cfg, *cache, first_layer, n_layers), Hq, n, (int)tiles, (int)split, dim, vectors, rotary ? rotary->amplitude : 1.f,
                           rotary ? rotary->freq : nullptr, (const uint16_t *)k_dev, (const uint16_t *)v_dev, (const uint16_t *)q_dev, (uint16_t *)q_out,
                           at_dev, count_dev, position_dev};
    const int turn = !dim ? TURN_NONE : rotary->layout == WNW_ROTARY_PAIRS ? TURN_PAIRS : dim % 16 ? TURN_HALVES_ODD : TURN_HALVES;
    paged_dispatch(*cfg, [&](auto d) {
        constexpr int DH = decltype(d)::value;
        auto *k = turn == TURN_NONE ? paged_append_kernel<DH, TURN_NONE> : turn == TURN_PAIRS ? paged_append_kernel<DH, TURN_PAIRS>
                  : turn == TURN_HALVES ? paged_append_kernel<DH, TURN_HALVES> : paged_append_kernel<DH, TURN_HALVES_ODD>;
        hipLaunchKernelGGL(k, dim3((unsigned)(tiles * layers * split)), dim3(P_THREADS), 0, (hipStream_t)hip_stream, a, TT);
    });
    return paged_hip();
}

wnw_status wnw_paged_keep(const wnw_paged_config *cfg, const wnw_paged_cache *cache, int32_t first_layer, int32_t n_layers, int32_t n,
                          const int32_t *base_dev, const int32_t *path_dev, const int32_t *count_dev, void *hip_stream)
{
    wnw_status st = paged_config(cfg, first_layer, n_layers, 0);
    if (st == WNW_OK) st = paged_cache(cache);
    if (st != WNW_OK) return st;
    if (n < 0) return paged_fail(WNW_ERR_INVALID, "negative n");
    if (n > 1024) return paged_fail(WNW_ERR_UNSUPPORTED, "paths of more than 1024 tokens");
    if (n == 0) return WNW_OK;
    if (!base_dev || !path_dev) return paged_fail(WNW_ERR_INVALID, "NULL pointer");
    if (off4(base_dev) || off4(path_dev) || off4(count_dev)) return paged_fail(WNW_ERR_INVALID, "a pointer is not aligned to its elements");
    const int items = 2 * cfg->batch * n_layers * cfg->kv_heads, per = P_THREADS / 64;
    const int64_t groups = ((int64_t)items + per - 1) / per;
    if (groups > P_MAX_GROUPS) return paged_fail(WNW_ERR_UNSUPPORTED, "too many heads for one call");
    const PagedGeo g = paged_geo(*cfg, *cache, first_layer, n_layers);
    paged_dispatch(*cfg, [&](auto d) {
        hipLaunchKernelGGL((paged_keep_kernel<decltype(d)::value>), dim3((unsigned)groups), dim3(P_THREADS), 0, (hipStream_t)hip_stream, g, n, items,
                           base_dev, path_dev, count_dev);
    });
    return paged_hip();
}

wnw_status wnw_paged_attend_workspace(const wnw_paged_config *cfg, int32_t n_layers, int32_t q_heads, int32_t n, int32_t max_len, size_t *bytes)
{
    wnw_status st = paged_config(cfg, 0, n_layers, n);
    if (st == WNW_OK) st = paged_heads(*cfg, n_layers, q_heads, n, max_len);
    if (st != WNW_OK) return st;
    if (!bytes) return paged_fail(WNW_ERR_INVALID, "NULL pointer");
    *bytes = n ? (size_t)paged_plan(*cfg, n_layers, q_heads, n, max_len).total() : 0;
    return WNW_OK;
}

wnw_status wnw_paged_attend(const wnw_paged_config *cfg, const wnw_paged_cache *cache, int32_t first_layer, int32_t n_layers, int32_t q_heads,
                            int32_t n, const void *q_dev, const int32_t *len_dev, const int32_t *count_dev, const uint64_t *mask_dev,
                            void *out_dev, float *lse_dev, int32_t max_len, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    wnw_status st = paged_config(cfg, first_layer, n_layers, n);
    if (st == WNW_OK) st = paged_cache(cache);
    if (st == WNW_OK) st = paged_heads(*cfg, n_layers, q_heads, n, max_len);
    if (st != WNW_OK) return st;
    if (n == 0) return WNW_OK;
    if (!q_dev || !len_dev || !out_dev) return paged_fail(WNW_ERR_INVALID, "NULL pointer");
    if (off16(q_dev) || off16(out_dev)) return paged_fail(WNW_ERR_INVALID, "queries and outputs must be aligned to 16 bytes");
    if (off4(len_dev) || off4(count_dev) || off4(lse_dev) || (uintptr_t)mask_dev & 7)
        return paged_fail(WNW_ERR_INVALID, "a pointer is not aligned to its elements");
    const PagedPlan p = paged_plan(*cfg, n_layers, q_heads, n, max_len);
    if (p.total() && (!workspace || off16(workspace) || workspace_bytes < (size_t)p.total()))
        return paged_fail(WNW_ERR_INVALID, "workspace missing, too small or not aligned to 16 bytes");
    const int G = q_heads / cfg->kv_heads, R = G * n;
    char *ws = (char *)workspace;
    const PagedAttend a = {paged_geo(*cfg, *cache, first_layer, n_layers), G, n, R, p.W, p.RB, __builtin_ctz((unsigned)p.RB), p.tsh,
                           cfg->flags & WNW_F_OUT_BF16 ? 1 : 0, p.whole ? (R + p.RB - 1) / p.RB : 0, 1.f / p.W, (const uint16_t *)q_dev, len_dev,
                           count_dev, (const unsigned long long *)mask_dev, out_dev, lse_dev, (float *)ws, (float2 *)(ws + p.o_bytes),
                           P_LOG2E / sqrtf((float)cfg->head_dim)};
    paged_dispatch(*cfg, [&](auto d) {
        constexpr int DH = decltype(d)::value;
        if (p.RB > 32)
            launch_wide<DH>(p, a, (hipStream_t)hip_stream);
        else if (p.RB == 32)
            launch_tokens<DH, 2>(p, a, (hipStream_t)hip_stream);
        else
            launch_tokens<DH, 1>(p, a, (hipStream_t)hip_stream);
        if (p.whole) return;
        const int per = p.join_groups ? 1 : 16;
        hipLaunchKernelGGL((p.join_groups ? paged_join_kernel<DH, 16> : paged_join_kernel<DH, 1>), dim3((unsigned)(p.rows / R * ((R + per - 1) / per))),
                           dim3(P_THREADS), 0, (hipStream_t)hip_stream, a);
    });
    return paged_hip();
}

}  // extern "C"
