// Drafted decoding apart from its cache: the tree of a draft, and which of its tokens stand.  Definitions as in wnw.h.
//
//   draft_tree_kernel    ancestors' bits and positions by doubling paths
//   draft_walk_kernel    the tokens that stand, a work-group per sequence
//   draft_slice_kernel   sums over 1024 tokens of what is left of the last row
//   draft_pick_kernel    the token that the last uniform number names
#include "wnw.h"
#include "wnw_parts.h"

#include <math.h>

#include <algorithm>
#include <cstring>

namespace wnw {

namespace {

constexpr int DRAFT_MAX = 1024;
constexpr int DRAFT_SLICE = 1024;   // tokens of a partial sum
constexpr int DRAFT_THREADS = 256;

// ---- the tree --------------------------------------------------------------------------------

// A work-group per sequence and word of the mask.  After r rounds a token knows the word's tokens among itself and the 2^r - 1
// before it on its path, how many of those there are, and which token comes before them all; a round joins a token with the one
// that its jump names, so that a path of m tokens takes log2(m) + 1 rounds.
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
struct Draft {
    int B, n, V, slices;
    const int32_t *token, *parent, *count;
    const float *target, *draft, *uniform;
    int32_t *path, *accepted, *next;
    double *t;           // [B] t of the last row
    int32_t *at;         // [B] the last token that stands, -1: none
    double *sums;        // [B][slices]
    __device__ size_t row(int b, int node) const { return ((size_t)b * (n + 1) + node + 1) * V; }
    __device__ int counted(int b) const { return count ? clamp_to(count[b], n) : n; }
    __device__ int parent_of(int b, int i) const
    {
        const int p = parent ? parent[(size_t)b * n + i] : i - 1;
        return p < 0 || p >= i ? -1 : p;
    }
};

__device__ inline double left_of(float p, float q, double t)
{
    return fmax((double)p - t * (double)q, 0.0);
}
__device__ inline double wave_sumd(double x)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s);
    return x;
}

__global__ __launch_bounds__(DRAFT_THREADS) void draft_walk_kernel(Draft d)
{
    __shared__ float sp[DRAFT_MAX], sq[DRAFT_MAX], su[DRAFT_MAX];
    __shared__ int from[DRAFT_MAX];
    __shared__ double part[DRAFT_THREADS / 64];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cnt = d.counted(b);
    for (int i = tid; i < d.n; i += DRAFT_THREADS) {
        float p = 0.f, q = 0.f;
        int f = -2;
        if (i < cnt) {
            const int x = d.token[(size_t)b * d.n + i];
            f = d.parent_of(b, i);
            if (x >= 0 && x < d.V) {
                p = d.target[d.row(b, f) + x];
                q = d.draft ? d.draft[d.row(b, f) + x] : 1.f;
            }
        }
        sp[i] = p, sq[i] = q, from[i] = f;
        su[i] = d.uniform[(size_t)b * (d.n + 1) + i];
        d.path[(size_t)b * d.n + i] = -1;
    }
    __syncthreads();
    // every wavefront takes the same steps
    int at = -1, stand = 0;
    double t = 0.0, s = 1.0;
    bool known = true;      // s is the sum for t
    for (int i0 = 0; i0 < cnt; i0 += 64) {
        unsigned long long left = ~0ull;
        for (;;) {
            // the next token that follows `at`
            const unsigned long long follow = __ballot(i0 + lane < cnt && from[min(i0 + lane, cnt - 1)] == at) & left;
            if (!follow) break;
            const int j = __builtin_ctzll(follow), i = i0 + j;
            left = j == 63 ? 0ull : ~0ull << (j + 1);
            if (!known) {
                const float *p = d.target + d.row(b, at), *q = d.draft + d.row(b, at);
                double x = 0.0;
                for (int v = tid; v < d.V; v += DRAFT_THREADS) x += left_of(p[v], q[v], t);
                x = wave_sumd(x);
                __syncthreads();
                if (lane == 0) part[wave] = x;
                __syncthreads();
                s = (part[0] + part[1]) + (part[2] + part[3]);
                known = true;
            }
            const double p = (double)sp[i], q = (double)sq[i], u = (double)su[i];
            if (d.draft ? u * q * s < fmax(p - t * q, 0.0) : u * s < p) {
                if (tid == 0) d.path[(size_t)b * d.n + stand] = i;
                ++stand;
                at = i, t = 0.0, s = 1.0;
            } else if (d.draft) {
                t += s;
                known = false;
            } else {
                // its token again, if another of the same follows, has nothing left
                s -= p;
                const int x = d.token[(size_t)b * d.n + i];
                __syncthreads();
                for (int k = i + 1 + tid; k < cnt; k += DRAFT_THREADS)
                    if (from[k] == at && d.token[(size_t)b * d.n + k] == x) sp[k] = 0.f;
                __syncthreads();
            }
        }
    }
    if (tid == 0) {
        d.accepted[b] = stand;
        d.at[b] = at;
        d.t[b] = t;
    }
}

// What is left of token v of the last row.  Without a draft's row, tokens that were refused there have nothing left.
struct LastRow {
    const float *p, *q;
    const int32_t *token;
    const Draft &d;
    int b, at, cnt;
    double t;
    __device__ LastRow(const Draft &d_, int b_) : d(d_), b(b_), at(d_.at[b_]), cnt(d_.counted(b_)), t(d_.t[b_])
    {
        p = d.target + d.row(b, at);
        q = d.draft ? d.draft + d.row(b, at) : nullptr;
        token = d.token + (size_t)b * d.n;
    }
    __device__ bool refused(int v) const
    {
        for (int i = at + 1; i < cnt; ++i)
            if (token[i] == v && d.parent_of(b, i) == at) return true;
        return false;
    }
    __device__ double operator()(int v, bool whole = false) const
    {
        if (whole) return fmax((double)p[v], 0.0);
        if (q) return t == 0.0 ? fmax((double)p[v], 0.0) : left_of(p[v], q[v], t);
        return refused(v) ? 0.0 : fmax((double)p[v], 0.0);
    }
};

__global__ __launch_bounds__(DRAFT_THREADS) void draft_slice_kernel(Draft d)
{
    const int item = blockIdx.x * (DRAFT_THREADS / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int b = item / d.slices, sl = item - b * d.slices;
    if (b >= d.B) return;
    const LastRow left(d, b);
    double x = 0.0;
    for (int v = sl * DRAFT_SLICE + lane; v < min(d.V, (sl + 1) * DRAFT_SLICE); v += 64) x += left(v);
    x = wave_sumd(x);
    if (lane == 0) d.sums[(size_t)b * d.slices + sl] = x;
}

__global__ __launch_bounds__(64) void draft_pick_kernel(Draft d)
{
    const int b = blockIdx.x, lane = threadIdx.x;
    const LastRow left(d, b);
    double *sums = d.sums + (size_t)b * d.slices;
    bool whole = false;
    double total;
    for (;;) {
        total = 0.0;
        for (int s = lane; s < d.slices; s += 64) total += sums[s];
        total = wave_sumd(total);
        if (total > 0.0 || whole) break;
        // nothing is left: the row itself
        whole = true;
        for (int s = 0; s < d.slices; ++s) {
            double x = 0.0;
            for (int v = s * DRAFT_SLICE + lane; v < min(d.V, (s + 1) * DRAFT_SLICE); v += 64) x += left(v, true);
            x = wave_sumd(x);
            if (lane == 0) sums[s] = x;
        }
        __syncthreads();
    }
    int got = -1;
    if (total > 0.0 && total < INFINITY) {
        const double goal = (double)d.uniform[(size_t)b * (d.n + 1) + d.n] * total;
        // the slice in which the running sum exceeds the goal, or the last one with anything left
        double run = 0.0, before = 0.0;
        int at = -1;
        for (int s = 0; s < d.slices; ++s) {
            const double x = sums[s];
            if (x > 0.0) at = s, before = run;
            run += x;
            if (x > 0.0 && run > goal) break;
        }
        run = before;
        for (int v0 = at * DRAFT_SLICE; v0 < min(d.V, (at + 1) * DRAFT_SLICE); v0 += 64) {
            const int v = v0 + lane;
            const double x = v < d.V ? left(v, whole) : 0.0;
            double sum = x;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) {
                const double y = __shfl_up(sum, s);
                if (lane >= s) sum += y;
            }
            const unsigned long long some = __ballot(x > 0.0), hit = __ballot(x > 0.0 && run + sum > goal);
            if (hit) {
                got = v0 + __builtin_ctzll(hit);
                break;
            }
            if (some) got = v0 + 63 - __builtin_clzll(some);
            run += __shfl(sum, 63);
        }
    }
    if (lane == 0) d.next[b] = got;
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
    if ((int64_t)batch * ((vocab + DRAFT_SLICE - 1) / DRAFT_SLICE) > (1 << 24))
        return draft_fail(WNW_ERR_UNSUPPORTED, "too many sequences for one call");
    return WNW_OK;
}
int slices_of(int32_t vocab)
{
    return (vocab + DRAFT_SLICE - 1) / DRAFT_SLICE;
}
size_t verify_bytes(int32_t batch, int32_t vocab)
{
    return (size_t)batch * (8 * (size_t)slices_of(vocab) + 8 + 4);
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
    hipLaunchKernelGGL(draft_tree_kernel, dim3((unsigned)(batch * words)), dim3((unsigned)words * 64), 0, (hipStream_t)hip_stream, n,
                       parent_dev, base_dev, count_dev, mask_dev, position_dev);
    return draft_hip();
}

wnw_status wnw_draft_verify_workspace(int32_t batch, int32_t n, int32_t vocab, size_t *bytes)
{
    const wnw_status st = verify_sizes(batch, n, vocab);
    if (st != WNW_OK) return st;
    if (!bytes) return draft_fail(WNW_ERR_INVALID, "NULL pointer");
    *bytes = verify_bytes(batch, vocab);
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
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < verify_bytes(batch, vocab))
        return draft_fail(WNW_ERR_INVALID, "workspace missing, too small or not aligned to 16 bytes");
    const int slices = slices_of(vocab);
    double *t = (double *)workspace, *sums = t + batch;
    const Draft d = {batch, n, vocab, slices, token_dev, parent_dev, count_dev, target_dev, draft_dev, uniform_dev,
                     path_dev, accepted_dev, next_dev, t, (int32_t *)(sums + (size_t)batch * slices), sums};
    const hipStream_t stream = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(draft_walk_kernel, dim3((unsigned)batch), dim3(DRAFT_THREADS), 0, stream, d);
    const int per = DRAFT_THREADS / 64;
    hipLaunchKernelGGL(draft_slice_kernel, dim3((unsigned)((batch * slices + per - 1) / per)), dim3(DRAFT_THREADS), 0, stream, d);
    hipLaunchKernelGGL(draft_pick_kernel, dim3((unsigned)batch), dim3(64), 0, stream, d);
    return draft_hip();
}

}  // extern "C"
