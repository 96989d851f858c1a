// Drafted decoding apart from its cache: the tree of a draft, and which of its tokens stand.  Definitions as in wnw.h.
//
//   draft_tree_kernel    ancestors' bits and positions by doubling paths
//   draft_round_kernel   a sum over the vocabulary that the tokens' verification needs, by slices
//   draft_verify_kernel  the tokens that stand and the one after them, a work-group per sequence
#include "wnw.h"
#include "wnw_parts.h"

#include <math.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

namespace wnw {

namespace {

constexpr int DRAFT_MAX = 1024;

// ---- the tree --------------------------------------------------------------------------------

// A work-group per sequence and word of the mask.  After r rounds a token knows the word's tokens among itself and the 2^r - 1
// before it on its path, how many of those there are, and which token comes before them all; a round joins a token with the one
// that its jump names, so that a path of m tokens takes log2(m) + 1 rounds.  Bound by latency: 16 tokens take 2.1 us, which is a launch;
// 16 sequences of 512 tokens in chains and branches 6.1 (a token that follows its parents one by one takes 512 dependent reads).
__global__ __launch_bounds__(DRAFT_MAX) void draft_tree_kernel(int n, const int32_t *__restrict__ parent, const int32_t *__restrict__ base,
                                                               const int32_t *__restrict__ count, uint64_t *__restrict__ mask,
                                                               int32_t *__restrict__ position)
{
    __shared__ uint64_t bits[DRAFT_MAX];
    __shared__ int jump[DRAFT_MAX], depth[DRAFT_MAX];
    const int words = (n + 63) / 64, b = blockIdx.x / words, w = blockIdx.x - b * words, i = threadIdx.x;
    const int cnt = count ? clamp_to(count[b], n) : n;
    uint64_t seen = 0;
    int from = -1, steps = 0;
    if (i < cnt) {
        from = parent[(size_t)b * n + i];
        if (from < 0 || from >= i) from = -1;
        seen = i >> 6 == w ? 1ull << (i & 63) : 0;
        steps = from >= 0 ? 1 : 0;
    }
    bits[i] = seen, jump[i] = from, depth[i] = steps;
    while (__syncthreads_or(from >= 0)) {
        const int at = from;
        if (at >= 0) {
            seen |= bits[at];
            steps += depth[at];
            from = jump[at];
        }
        __syncthreads();
        bits[i] = seen, jump[i] = from, depth[i] = steps;
    }
    if (i >= cnt) return;
    if (mask) mask[((size_t)b * n + i) * words + w] = seen;
    if (position && w == 0) position[(size_t)b * n + i] = base[b] + steps;
}

// ---- verification ----------------------------------------------------------------------------

// With t_0 = 0, s_0 = 1, t_{k+1} = t_k + s_k and s_k = sum of max(p - t_k q, 0) for k > 0, what is left of p after k refused
// tokens is max(p - t_k q, 0) / s_k, since max(max(x, 0) - q, 0) = max(x - q, 0) for q >= 0.  So a refused token costs one sum over
// the vocabulary, and only where another one is tried after it.
//
// A sum over the vocabulary is one compute unit's work for 9 us (131072 tokens) where a work-group has a sequence, so for large
// vocabularies and few sequences some launches go in front (draft_round_kernel) in which every sequence has a work-group for each
// slice of the vocabulary: all of them walk to the next sum that is needed and leave their slice's part of it.  Rounds that a sequence
// does not need end at once; sums that no round was there for are taken by its one work-group at the end (draft_verify_kernel), which also
// finds the token after the path: the slices' sums name the slice that the last uniform number falls into, and a scan of that one the token.
// Bound by latency, as one sum needs the one before it: five tokens one after the other, 32000 tokens in the vocabulary, 10.5 us; eight
// trees of 64 tokens, 131072 in the vocabulary, 30 to 42 us by the number of sums that the random numbers ask for, 4 to 5.2 us each (357 with one
// work-group for a sequence and a sum for every token).
constexpr int ROUND_THREADS = 256, VERIFY_THREADS = 1024;
constexpr int MAX_SLICES = 2048, ROUND_SLICES = 64;

// How far a sequence is along its path.
struct DraftState {
    double t, s;       // of the row behind `at`; s is the sum for t if `known`
    int at, stand;     // the last token that stands (-1: none), how many do
    int i, known;      // tokens before i have been tried
    int phase;         // what the sums that come next are for
    int sums;          // the round that has them
};
enum { NEED_SUM, NEED_TOTAL, HAVE_TOTAL };

struct Draft {
    int n, V, slice, slices;     // slice: tokens of a partial sum, a multiple of 1024
    int rounds;
    const int32_t *token, *parent, *count;
    const float *target, *draft, *uniform;
    int32_t *path, *accepted, *next;
    DraftState *state;           // [2][B], by turns
    double *sums;                // [B][rounds][slices]
    float2 *pq;                  // [B][n] the tokens' probabilities, and what they follow and are, from the first round for later ones
    int2 *link;
    __device__ double *sums_of(int b, int round) const { return sums + ((size_t)b * rounds + round) * slices; }
};

__device__ inline double wave_sumd(double x)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s);
    return x;
}
__device__ inline double wave_scand(double x, int lane)
{
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const double y = __shfl_up(x, s);
        if (lane >= s) x += y;
    }
    return x;
}

typedef float df4_t __attribute__((ext_vector_type(4)));

// What is left of four tokens' p.
template <bool Q>
__device__ inline double left4(df4_t p, df4_t q, double t)
{
    double x = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) x += Q ? fmax((double)p[e] - t * (double)q[e], 0.0) : fmax((double)p[e], 0.0);
    return x;
}
// The sum over tokens v0 .. v1 - 1, by `threads` threads of which this is number i; rows at 16 bytes (VEC) or any fp32 address.
template <bool Q, bool VEC>
__device__ inline double left_sum(const float *p, const float *q, double t, int v0, int v1, int i, int threads)
{
    double x = 0.0;
    if constexpr (VEC) {
#pragma unroll 4
        for (int v = v0 + 4 * i; v < v1; v += 4 * threads)
            x += left4<Q>(*(const df4_t *)(p + v), Q ? *(const df4_t *)(q + v) : df4_t{}, t);
    } else {
#pragma unroll 8
        for (int v = v0 + i; v < v1; v += threads) x += Q ? fmax((double)p[v] - t * (double)q[v], 0.0) : fmax((double)p[v], 0.0);
    }
    return x;
}

// A sequence's drafted tokens, with their probabilities behind their parents.
struct DraftTokens {
    float p[DRAFT_MAX], q[DRAFT_MAX], u[DRAFT_MAX];
    int from[DRAFT_MAX], token[DRAFT_MAX];
    int refused;                            // tokens refused at the last row, then in `token`

    // again: a round has been here.  (All n tokens, so that nothing waits for the count.)
    __device__ void load(const Draft &d, int b, int threads, bool again, bool keep)
    {
        const int n = d.n, V = d.V;
        if (again) {
            for (int i = threadIdx.x; i < n; i += threads) {
                const float2 x = d.pq[(size_t)b * n + i];
                const int2 y = d.link[(size_t)b * n + i];
                p[i] = x.x, q[i] = x.y, from[i] = y.x, token[i] = y.y, u[i] = d.uniform[(size_t)b * (n + 1) + i];
            }
            if (threadIdx.x == 0) refused = 0;
            __syncthreads();
            return;
        }
        const float *target = d.target + (size_t)b * (n + 1) * V, *draft = d.draft ? d.draft + (size_t)b * (n + 1) * V : nullptr;
        for (int i = threadIdx.x; i < n; i += threads) {
            const int x = d.token[(size_t)b * n + i];
            int f = d.parent ? d.parent[(size_t)b * n + i] : i - 1;
            if (f < 0 || f >= i) f = -1;
            float pp = 0.f, qq = 0.f;
            if (x >= 0 && x < V) {
                const size_t at = (size_t)(f + 1) * V + x;
                pp = target[at];
                qq = draft ? draft[at] : 1.f;
            }
            p[i] = pp, q[i] = qq, u[i] = d.uniform[(size_t)b * (n + 1) + i], from[i] = f, token[i] = x;
            if (keep) d.pq[(size_t)b * n + i] = make_float2(pp, qq), d.link[(size_t)b * n + i] = make_int2(f, x);
        }
        if (threadIdx.x == 0) refused = 0;
        __syncthreads();
    }
    // On to the next sum that is needed; every wavefront takes the same steps.  path: where the tokens that stand go (one work-group's), or null.
    __device__ void walk(const Draft &d, DraftState &st, int cnt, int32_t *path)
    {
        const int tid = threadIdx.x, lane = tid & 63;
        for (int i0 = st.i & ~63; i0 < cnt; i0 += 64) {
            unsigned long long later = st.i > i0 ? ~0ull << (st.i & 63) : ~0ull;
            for (;;) {
                // the next token that follows `at`
                const unsigned long long follow = __ballot(i0 + lane < cnt && from[min(i0 + lane, cnt - 1)] == st.at) & later;
                if (!follow) break;
                const int j = __builtin_ctzll(follow), i = i0 + j;
                later = j == 63 ? 0ull : ~0ull << (j + 1);
                if (!st.known) {
                    st.i = i, st.phase = NEED_SUM;
                    return;
                }
                const double pp = (double)p[i], qq = (double)q[i], uu = (double)u[i];
                if (d.draft ? uu * qq * st.s < fmax(st.t == 0.0 ? pp : pp - st.t * qq, 0.0) : uu * st.s < pp) {
                    if (path && tid == 0) path[st.stand] = i;
                    ++st.stand;
                    st.at = i, st.t = 0.0, st.s = 1.0;
                } else if (d.draft) {
                    st.t += st.s;
                    st.known = 0;
                } else {
                    // its token again, if another of the same follows, has nothing left
                    st.s -= fmax(pp, 0.0);
                    const int x = token[i];
                    __syncthreads();
                    for (int k = i + 1 + tid; k < cnt; k += blockDim.x)
                        if (from[k] == st.at && token[k] == x) p[k] = 0.f;
                    __syncthreads();
                }
            }
        }
        st.i = cnt, st.phase = NEED_TOTAL;
    }
    // The tokens refused at the last row that lie in v0 .. v1 - 1 to the front of `token` (in any order: they are only looked up).
    __device__ void collect(int cnt, int at, int v0, int v1, int threads)
    {
        for (int i0 = 0; i0 < cnt; i0 += threads) {
            const int i = i0 + threadIdx.x, x = i < cnt ? token[i] : -1;
            const bool is = i < cnt && from[i] == at && x >= v0 && x < v1;
            __syncthreads();
            if (is) token[atomicAdd(&refused, 1)] = x;      // (entries below i0 + threads only, all of them read)
        }
        __syncthreads();
    }
    __device__ bool has_refused(int v) const
    {
        for (int k = 0; k < refused; ++k)
            if (token[k] == v) return true;
        return false;
    }
};

// A round: the part that slice blockIdx.x of the vocabulary has in the next sum of sequence blockIdx.y.
template <bool VEC>
__global__ __launch_bounds__(ROUND_THREADS) void draft_round_kernel(Draft d, int round)
{
    __shared__ DraftTokens tokens;
    __shared__ double part[ROUND_THREADS / 64];
    const int g = blockIdx.x, b = blockIdx.y, B = gridDim.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int cnt = d.count ? clamp_to(d.count[b], d.n) : d.n;
    DraftState st = {0.0, 1.0, -1, 0, 0, 1, NEED_SUM, 0};
    double sum = 0.0;
    if (round) {
        // (before the state decides, so that all that was left is fetched at once)
        st = d.state[(size_t)(round - 1 & 1) * B + b];
        if (lane < d.slices) sum = d.sums_of(b, round - 1)[lane];
    }
    tokens.load(d, b, ROUND_THREADS, round > 0, round == 0 && g == 0);
    if (round) {
        if (st.phase == NEED_TOTAL) st.phase = HAVE_TOTAL;
        if (st.phase == HAVE_TOTAL) {
            if (g == 0 && tid == 0) d.state[(size_t)(round & 1) * B + b] = st;
            return;
        }
        st.s = wave_sumd(sum);
        st.known = 1;
    }
    int32_t *path = d.path + (size_t)b * d.n;
    if (!round && g == 0) {
        for (int i = tid; i < d.n; i += ROUND_THREADS) path[i] = -1;
        __syncthreads();
    }
    tokens.walk(d, st, cnt, g == 0 ? path : nullptr);
    st.sums = round;
    if (g == 0 && tid == 0) d.state[(size_t)(round & 1) * B + b] = st;

    const size_t row = ((size_t)b * (d.n + 1) + st.at + 1) * d.V;
    const float *p = d.target + row, *q = d.draft && st.t > 0.0 ? d.draft + row : nullptr;
    const int v0 = g * d.slice, v1 = min(d.V, v0 + d.slice);
    double x = 0.0;
    if (!d.draft) tokens.collect(cnt, st.at, v0, v1, ROUND_THREADS);
    if (tokens.refused) {
        for (int v = v0 + tid; v < v1; v += ROUND_THREADS) x += tokens.has_refused(v) ? 0.0 : fmax((double)p[v], 0.0);
    } else if (q)
        x = left_sum<true, VEC>(p, q, st.t, v0, v1, tid, ROUND_THREADS);
    else
        x = left_sum<false, VEC>(p, nullptr, 0.0, v0, v1, tid, ROUND_THREADS);
    x = wave_sumd(x);
    if (lane == 0) part[wave] = x;
    __syncthreads();
    if (tid == 0) d.sums_of(b, round)[g] = (part[0] + part[1]) + (part[2] + part[3]);
}

struct VerifySmem {
    DraftTokens tokens;
    double sums[MAX_SLICES];
    double part[VERIFY_THREADS / 64];
    unsigned marked[MAX_SLICES / 32];       // slices with a refused token
    int first[VERIFY_THREADS / 64], last[VERIFY_THREADS / 64], got, found;
};

template <bool VEC>
__global__ __launch_bounds__(VERIFY_THREADS) void draft_verify_kernel(Draft d)
{
    __shared__ VerifySmem sm;
    constexpr int WAVES = VERIFY_THREADS / 64;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = d.n, V = d.V, slice = d.slice, slices = d.slices;
    const int cnt = d.count ? clamp_to(d.count[b], n) : n;
    const float chosen = d.uniform[(size_t)b * (n + 1) + n];
    int32_t *path = d.path + (size_t)b * n;
    DraftState st = {0.0, 1.0, -1, 0, 0, 1, NEED_SUM, 0};
    if (d.rounds) {
        st = d.state[(size_t)(d.rounds - 1 & 1) * gridDim.x + b];
        if (st.phase == NEED_TOTAL) st.phase = HAVE_TOTAL;
        for (int k = tid; k < slices; k += VERIFY_THREADS) sm.sums[k] = d.sums_of(b, st.sums)[k];
    }
    sm.tokens.load(d, b, VERIFY_THREADS, d.rounds > 0, false);
    if (tid < MAX_SLICES / 32) sm.marked[tid] = 0;
    if (tid == 0) sm.got = -1, sm.found = 0;
    if (!d.rounds && tid < n) path[tid] = -1;
    __syncthreads();
    if (st.phase == NEED_SUM) {
        if (d.rounds) {
            st.s = wave_sumd(lane < slices ? sm.sums[lane] : 0.0);
            st.known = 1;
            __syncthreads();
        }
        for (;;) {
            sm.tokens.walk(d, st, cnt, path);
            if (st.phase == NEED_TOTAL) break;
            const size_t row = ((size_t)b * (n + 1) + st.at + 1) * V;
            const double x = wave_sumd(left_sum<true, VEC>(d.target + row, d.draft + row, st.t, 0, V, tid, VERIFY_THREADS));
            if (lane == 0) sm.part[wave] = x;
            __syncthreads();
            st.s = 0.0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) st.s += sm.part[w];
            st.known = 1;
            __syncthreads();
        }
    }
    if (tid == 0) d.accepted[b] = st.stand;

    // the token after them
    const size_t row = ((size_t)b * (n + 1) + st.at + 1) * V;
    const float *p = d.target + row, *q = d.draft && st.t > 0.0 ? d.draft + row : nullptr;
    if (!d.draft) {
        sm.tokens.collect(cnt, st.at, 0, V, VERIFY_THREADS);
        for (int k = tid; k < sm.tokens.refused; k += VERIFY_THREADS)
            atomicOr(&sm.marked[sm.tokens.token[k] / slice >> 5], 1u << (sm.tokens.token[k] / slice & 31));
        __syncthreads();
    }
    // of token v; whole: of the row as it is
    auto left = [&](int v, bool whole) {
        const double x = (double)p[v];
        if (whole) return fmax(x, 0.0);
        if (q) return fmax(x - st.t * (double)q[v], 0.0);
        return sm.tokens.has_refused(v) ? 0.0 : fmax(x, 0.0);
    };
    bool whole = false;
    double total;
    for (;;) {
        if (st.phase != HAVE_TOTAL || whole)
            for (int k = wave; k < slices; k += WAVES) {
                const int v0 = k * slice, v1 = min(V, v0 + slice);
                double x;
                if (!whole && sm.marked[k >> 5] >> (k & 31) & 1) {
                    x = 0.0;
                    for (int v = v0 + lane; v < v1; v += 64) x += left(v, false);
                } else if (q && !whole)
                    x = left_sum<true, VEC>(p, q, st.t, v0, v1, lane, 64);
                else
                    x = left_sum<false, VEC>(p, nullptr, 0.0, v0, v1, lane, 64);
                x = wave_sumd(x);
                if (lane == 0) sm.sums[k] = x;
            }
        __syncthreads();
        total = 0.0;
        for (int k = lane; k < slices; k += 64) total += sm.sums[k];
        total = wave_sumd(total);
        if (total > 0.0 || whole) break;
        whole = true;       // nothing is left: the row itself
        __syncthreads();
    }
    if (!(total > 0.0 && total < INFINITY)) {
        if (tid == 0) d.next[b] = -1;
        return;
    }
    const double goal = (double)chosen * total;
    // the slice in which the running sum exceeds the goal, or the last one with anything left; every wavefront finds it
    int in = -1;
    double run = 0.0, before = 0.0;
    for (int k0 = 0; k0 < slices; k0 += 64) {
        const double x = k0 + lane < slices ? sm.sums[k0 + lane] : 0.0, sum = run + wave_scand(x, lane);
        const unsigned long long some = __ballot(x > 0.0), hit = __ballot(x > 0.0 && sum > goal);
        const int j = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : -1;
        if (j >= 0) in = k0 + j, before = __shfl(sum - x, j);
        if (hit) break;
        run = __shfl(sum, 63);
    }
    // in it, the first token at which it does, or the last one with anything left; E tokens a thread
    const int end = min(V, (in + 1) * slice);
    auto scan = [&](auto each) {
        constexpr int E = decltype(each)::value;
        for (int v0 = in * slice; v0 < end; v0 += E * VERIFY_THREADS) {
            const int v = v0 + E * tid;
            float ps[E] = {}, qs[E] = {};
            if constexpr (VEC && E == 4) {
                if (v < end) {
                    __builtin_memcpy(ps, __builtin_assume_aligned(p + v, 16), sizeof(ps));
                    if (q && !whole) __builtin_memcpy(qs, __builtin_assume_aligned(q + v, 16), sizeof(qs));
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (v + e < end) {
                        ps[e] = p[v + e];
                        if (q && !whole) qs[e] = q[v + e];
                    }
            }
            double x[E], sum = 0.0;      // what is left of each; of all of them
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = fmax((double)ps[e] - st.t * (double)qs[e], 0.0);
                if (!whole && sm.tokens.refused && sm.tokens.has_refused(v + e)) x[e] = 0.0;
                sum += x[e];
            }
            const double upto = wave_scand(sum, lane);
            if (lane == 63) sm.part[wave] = upto;
            __syncthreads();
            double mine = __shfl_up(upto, 1);
            mine = before + (lane ? mine : 0.0);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) mine += sm.part[w];
                before += sm.part[w];
            }
            int first = -1, last = -1;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                mine += x[e];
                if (x[e] > 0.0) {
                    last = v + e;
                    if (first < 0 && mine > goal) first = v + e;
                }
            }
            const unsigned long long some = __ballot(last >= 0), hit = __ballot(first >= 0);
            first = hit ? __shfl(first, __builtin_ctzll(hit)) : -1;
            last = some ? __shfl(last, 63 - __builtin_clzll(some)) : -1;
            if (lane == 0) sm.first[wave] = first, sm.last[wave] = last;
            __syncthreads();
            if (tid == 0) {
                last = -1;
                for (int w = WAVES - 1; w >= 0; --w) {
                    if (sm.first[w] >= 0) sm.got = sm.first[w], sm.found = 1;
                    if (last < 0) last = sm.last[w];
                }
                if (!sm.found && last >= 0) sm.got = last;
            }
            __syncthreads();
            if (sm.found) break;
        }
    };
    // (slices of 1024 are one step with a token each already)
    slice > VERIFY_THREADS ? scan(std::integral_constant<int, 4>{}) : scan(std::integral_constant<int, 1>{});
    if (tid == 0) d.next[b] = sm.got;
}

// ---- host ------------------------------------------------------------------------------------

thread_local char d_msg[256] = "no error";

wnw_status draft_fail(wnw_status st, const char *msg)
{
    strncpy(d_msg, msg, sizeof d_msg - 1);
    return st;
}
wnw_status draft_hip()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WNW_OK : draft_fail(WNW_ERR_HIP, hipGetErrorString(e));
}
wnw_status draft_sizes(int32_t batch, int32_t n)
{
    if (batch < 1) return draft_fail(WNW_ERR_INVALID, "batch must be at least 1");
    if (n < 0) return draft_fail(WNW_ERR_INVALID, "negative n");
    if (n > DRAFT_MAX) return draft_fail(WNW_ERR_UNSUPPORTED, "more than 1024 drafted tokens");
    if (batch > (1 << 20)) return draft_fail(WNW_ERR_UNSUPPORTED, "more than 2^20 sequences");
    return WNW_OK;
}
wnw_status verify_sizes(int32_t batch, int32_t n, int32_t vocab)
{
    const wnw_status st = draft_sizes(batch, n);
    if (st != WNW_OK) return st;
    if (vocab < 1) return draft_fail(WNW_ERR_INVALID, "vocab must be at least 1");
    if (vocab > (1 << 24)) return draft_fail(WNW_ERR_UNSUPPORTED, "more than 2^24 tokens in the vocabulary");
    return WNW_OK;
}
// What sums a verification takes: the last row's alone (tokens one after the other), some on the way (a tree whose tokens were drawn),
// or the last row's without the tokens that were refused (tokens that were chosen).
enum VerifyKind { VERIFY_CHAIN, VERIFY_TREE, VERIFY_CHOSEN };

// Launches in front of the last one, 4 us each (2 us where a sequence has no more sums).  Measured without them and with: five tokens one
// after the other, 32000 tokens in the vocabulary, one sequence 10.7 and 10.9 us, 50000 12.2 and 11.0, 131072 18.6 and 13.9, 65536
// and 32 sequences 15.3 and 16.9; trees of 16, 50000, one sequence 16.6 and (three) 17.3, 131072 32.8 and 21.5, eight sequences 50.7
// and (five) 32.1, 65536 and 32 sequences 33 and 35; chosen tokens, 16384, one sequence 15.4 and 13.3, 131072, eight 27.7 and 18.1.
int verify_rounds(int32_t batch, int32_t vocab, VerifyKind kind)
{
    if (kind == VERIFY_CHOSEN) return vocab >= 16384 && batch <= 32 ? 1 : 0;
    if (batch > 16) return 0;
    if (kind == VERIFY_CHAIN) return vocab >= 49152 ? 1 : 0;
    return vocab >= 65536 ? (batch > 2 ? 5 : 3) : 0;
}
struct VerifyPlan {
    int slice, slices, rounds;
    size_t state_bytes, sum_bytes, token_bytes, bytes;
};
VerifyPlan verify_plan(int32_t batch, int32_t n, int32_t vocab, VerifyKind kind)
{
    VerifyPlan p;
    p.rounds = verify_rounds(batch, vocab, kind);
    const int most = p.rounds ? ROUND_SLICES : MAX_SLICES;
    p.slice = std::max(1024, (vocab + most * 1024 - 1) / (most * 1024) * 1024);
    p.slices = (vocab + p.slice - 1) / p.slice;
    p.state_bytes = p.rounds ? 2 * batch * sizeof(DraftState) : 0;
    p.sum_bytes = (size_t)batch * p.rounds * p.slices * sizeof(double);
    p.token_bytes = p.rounds ? (size_t)batch * n * sizeof(float2) : 0;
    p.bytes = p.state_bytes + p.sum_bytes + 2 * p.token_bytes;
    return p;
}
size_t verify_bytes(int32_t batch, int32_t n, int32_t vocab)
{
    size_t most = 0;
    for (const VerifyKind k : {VERIFY_CHAIN, VERIFY_TREE, VERIFY_CHOSEN}) most = std::max(most, verify_plan(batch, n, vocab, k).bytes);
    return most;
}
bool misaligned(const void *p, uintptr_t to)
{
    return (uintptr_t)p & (to - 1);
}

}  // namespace

}  // namespace wnw

using namespace wnw;

extern "C" {

const char *wnw_draft_last_error(void)
{
    return d_msg;
}

wnw_status wnw_draft_tree(int32_t batch, int32_t n, const int32_t *parent_dev, const int32_t *base_dev, const int32_t *count_dev,
                          uint64_t *mask_dev, int32_t *position_dev, void *hip_stream)
{
    const wnw_status st = draft_sizes(batch, n);
    if (st != WNW_OK) return st;
    if (n == 0 || (!mask_dev && !position_dev)) return WNW_OK;
    if (!parent_dev || (position_dev && !base_dev)) return draft_fail(WNW_ERR_INVALID, "NULL pointer");
    if (misaligned(parent_dev, 4) || misaligned(base_dev, 4) || misaligned(count_dev, 4) || misaligned(mask_dev, 8) || misaligned(position_dev, 4))
        return draft_fail(WNW_ERR_INVALID, "a pointer is not aligned to its elements");
    const int words = (n + 63) / 64;
    if ((int64_t)batch * words * words * 64 > 0xffffffffll) return draft_fail(WNW_ERR_UNSUPPORTED, "too many tokens for one call");
    hipLaunchKernelGGL(draft_tree_kernel, dim3((unsigned)(batch * words)), dim3((unsigned)words * 64), 0, (hipStream_t)hip_stream, n,
                       parent_dev, base_dev, count_dev, mask_dev, position_dev);
    return draft_hip();
}

wnw_status wnw_draft_verify_workspace(int32_t batch, int32_t n, int32_t vocab, size_t *bytes)
{
    const wnw_status st = verify_sizes(batch, n, vocab);
    if (st != WNW_OK) return st;
    if (!bytes) return draft_fail(WNW_ERR_INVALID, "NULL pointer");
    *bytes = verify_bytes(batch, n, vocab);
    return WNW_OK;
}

wnw_status wnw_draft_verify(int32_t batch, int32_t n, int32_t vocab, const int32_t *token_dev, const int32_t *parent_dev,
                            const int32_t *count_dev, const float *target_dev, const float *draft_dev, const float *uniform_dev,
                            int32_t *path_dev, int32_t *accepted_dev, int32_t *next_dev, void *workspace, size_t workspace_bytes,
                            void *hip_stream)
{
    const wnw_status st = verify_sizes(batch, n, vocab);
    if (st != WNW_OK) return st;
    if (!target_dev || !uniform_dev || !accepted_dev || !next_dev || (n > 0 && (!token_dev || !path_dev)))
        return draft_fail(WNW_ERR_INVALID, "NULL pointer");
    const void *all[] = {token_dev, parent_dev, count_dev, target_dev, draft_dev, uniform_dev, path_dev, accepted_dev, next_dev};
    for (const void *p : all)
        if (misaligned(p, 4)) return draft_fail(WNW_ERR_INVALID, "a pointer is not aligned to its elements");
    if (const size_t need = verify_bytes(batch, n, vocab); need && (!workspace || misaligned(workspace, 16) || workspace_bytes < need))
        return draft_fail(WNW_ERR_INVALID, "workspace missing, too small or not aligned to 16 bytes");
    const VerifyPlan p = verify_plan(batch, n, vocab, n <= 1 || (draft_dev && !parent_dev) ? VERIFY_CHAIN : draft_dev ? VERIFY_TREE : VERIFY_CHOSEN);
    char *ws = (char *)workspace;
    const Draft d = {n, vocab, p.slice, p.slices, p.rounds, token_dev, parent_dev, count_dev, target_dev, draft_dev, uniform_dev, path_dev, accepted_dev,
                     next_dev, (DraftState *)workspace, (double *)(ws + p.state_bytes), (float2 *)(ws + p.state_bytes + p.sum_bytes),
                     (int2 *)(ws + p.state_bytes + p.sum_bytes + p.token_bytes)};
    const bool vec = vocab % 4 == 0 && !misaligned(target_dev, 16) && !misaligned(draft_dev, 16);
    for (int r = 0; r < p.rounds; ++r)
        hipLaunchKernelGGL(vec ? draft_round_kernel<true> : draft_round_kernel<false>, dim3((unsigned)p.slices, (unsigned)batch), dim3(ROUND_THREADS), 0,
                           (hipStream_t)hip_stream, d, r);
    hipLaunchKernelGGL(vec ? draft_verify_kernel<true> : draft_verify_kernel<false>, dim3((unsigned)batch), dim3(VERIFY_THREADS), 0,
                       (hipStream_t)hip_stream, d);
    return draft_hip();
}

}  // extern "C"
