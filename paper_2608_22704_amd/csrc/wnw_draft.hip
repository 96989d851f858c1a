// Drafted decoding apart from its cache: the tree of a draft, and which of its tokens stand.  Definitions as in wnw.h.
//
//   draft_tree_kernel    ancestors' bits and positions by doubling paths
//   draft_verify_kernel  the tokens that stand and the one after them, a work-group per sequence
#include "wnw.h"
#include "wnw_parts.h"

#include <math.h>

#include <algorithm>
#include <cstring>

namespace wnw {

namespace {

constexpr int DRAFT_MAX = 1024;

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
//
// A work-group has a sequence: the drafted tokens' probabilities come first, all at once; then all of its wavefronts take the same
// steps along the path, and the sums by slices of the vocabulary; at the end the slices' sums name the slice that the last
// uniform number falls into, and a scan of that one the token.
constexpr int VERIFY_THREADS = 1024;
constexpr int MAX_SLICES = 2048;

struct Draft {
    int n, V, slice;     // slice: tokens of a partial sum, a multiple of 1024
    const int32_t *token, *parent, *count;
    const float *target, *draft, *uniform;
    int32_t *path, *accepted, *next;
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

struct VerifySmem {
    double sums[MAX_SLICES];
    double part[VERIFY_THREADS / 64];
    unsigned marked[MAX_SLICES / 32];       // slices with a refused token
    float p[DRAFT_MAX], q[DRAFT_MAX], u[DRAFT_MAX];
    int from[DRAFT_MAX], token[DRAFT_MAX];
    int refused;                            // tokens refused at the last row, then in `token`
    int got;
};

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

template <bool VEC>
__global__ __launch_bounds__(VERIFY_THREADS) void draft_verify_kernel(Draft d)
{
    __shared__ VerifySmem sm;
    constexpr int WAVES = VERIFY_THREADS / 64;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = d.n, V = d.V;
    const int cnt = d.count ? clamp_to(d.count[b], n) : n;
    const float *target = d.target + (size_t)b * (n + 1) * V, *draft = d.draft ? d.draft + (size_t)b * (n + 1) * V : nullptr;
    const float *uniform = d.uniform + (size_t)b * (n + 1);
    if (tid < n) {
        float p = 0.f, q = 0.f;
        int f = -2, x = -1;
        if (tid < cnt) {
            x = d.token[(size_t)b * n + tid];
            f = d.parent ? d.parent[(size_t)b * n + tid] : tid - 1;
            if (f < 0 || f >= tid) f = -1;
            if (x >= 0 && x < V) {
                const size_t at = (size_t)(f + 1) * V + x;
                p = target[at];
                q = draft ? draft[at] : 1.f;
            }
        }
        sm.p[tid] = p, sm.q[tid] = q, sm.u[tid] = uniform[tid], sm.from[tid] = f, sm.token[tid] = x;
        d.path[(size_t)b * n + tid] = -1;
    }
    if (tid < MAX_SLICES / 32) sm.marked[tid] = 0;
    if (tid == 0) sm.refused = 0, sm.got = -1;
    __syncthreads();

    // the path
    int at = -1, stand = 0;
    double t = 0.0, s = 1.0;
    bool known = true;      // s is the sum for t
    for (int i0 = 0; i0 < cnt; i0 += 64) {
        unsigned long long later = ~0ull;
        for (;;) {
            const unsigned long long follow = __ballot(i0 + lane < cnt && sm.from[min(i0 + lane, cnt - 1)] == at) & later;
            if (!follow) break;
            const int j = __builtin_ctzll(follow), i = i0 + j;
            later = j == 63 ? 0ull : ~0ull << (j + 1);
            if (!known) {
                const double x = wave_sumd(left_sum<true, VEC>(target + (size_t)(at + 1) * V, draft + (size_t)(at + 1) * V, t, 0, V, tid, VERIFY_THREADS));
                __syncthreads();
                if (lane == 0) sm.part[wave] = x;
                __syncthreads();
                s = 0.0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) s += sm.part[w];
                known = true;
            }
            const double p = (double)sm.p[i], q = (double)sm.q[i], u = (double)sm.u[i];
            if (draft ? u * q * s < fmax(t == 0.0 ? p : p - t * q, 0.0) : u * s < p) {
                if (tid == 0) d.path[(size_t)b * n + stand] = i;
                ++stand;
                at = i, t = 0.0, s = 1.0;
            } else if (draft) {
                t += s;
                known = false;
            } else {
                // its token again, if another of the same follows, has nothing left
                s -= fmax(p, 0.0);
                const int x = sm.token[i];
                __syncthreads();
                if (tid > i && tid < cnt && sm.from[tid] == at && sm.token[tid] == x) sm.p[tid] = 0.f;
                __syncthreads();
            }
        }
    }
    if (tid == 0) d.accepted[b] = stand;

    // the token after it
    const float *p = target + (size_t)(at + 1) * V, *q = draft && t > 0.0 ? draft + (size_t)(at + 1) * V : nullptr;
    const int slice = d.slice, slices = (V + slice - 1) / slice;
    if (!draft) {
        const int x = tid < cnt ? sm.token[tid] : -1;
        const bool refused = tid < cnt && sm.from[tid] == at && x >= 0 && x < V;
        __syncthreads();
        if (refused) {
            sm.token[atomicAdd(&sm.refused, 1)] = x;        // (in any order: they are only looked up)
            atomicOr(&sm.marked[x / slice >> 5], 1u << (x / slice & 31));
        }
        __syncthreads();
    }
    // of token v; whole: of the row as it is
    auto left = [&](int v, bool whole) {
        const double x = (double)p[v];
        if (whole) return fmax(x, 0.0);
        if (q) return fmax(x - t * (double)q[v], 0.0);
        for (int k = 0; k < sm.refused; ++k)
            if (sm.token[k] == v) return 0.0;
        return fmax(x, 0.0);
    };
    bool whole = false;
    double total;
    for (;;) {
        for (int k = wave; k < slices; k += WAVES) {
            const int v0 = k * slice, v1 = min(V, v0 + slice);
            double x;
            if (!whole && sm.marked[k >> 5] >> (k & 31) & 1) {
                x = 0.0;
                for (int v = v0 + lane; v < v1; v += 64) x += left(v, false);
            } else if (q && !whole)
                x = left_sum<true, VEC>(p, q, t, v0, v1, lane, 64);
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
    const double goal = (double)uniform[n] * total;
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
    for (int v0 = in * slice; v0 < min(V, (in + 1) * slice); v0 += VERIFY_THREADS) {
        const int v = v0 + tid;
        const double x = v < V ? left(v, whole) : 0.0;
        const double sum = wave_scand(x, lane);
        __syncthreads();
        if (lane == 63) sm.part[wave] = sum;
        __syncthreads();
        double mine = before;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) mine = before + sum;
            before += sm.part[w];
        }
        // the first that exceeds the goal, or the last one with anything left
        const unsigned long long some = __ballot(x > 0.0), hit = __ballot(x > 0.0 && mine > goal);
        __syncthreads();
        int *mark = (int *)sm.sums;
        if (lane == 0) {
            mark[wave] = hit ? v0 + wave * 64 + __builtin_ctzll(hit) : -1;
            mark[WAVES + wave] = some ? v0 + wave * 64 + 63 - __builtin_clzll(some) : -1;
        }
        __syncthreads();
        if (tid == 0) {
            int first = -1, last = -1;
            for (int w = WAVES - 1; w >= 0; --w) {
                if (mark[w] >= 0) first = mark[w];
                if (last < 0) last = mark[WAVES + w];
            }
            if (first >= 0)
                sm.got = first, sm.refused = -1;
            else if (last >= 0)
                sm.got = last;
        }
        __syncthreads();
        if (sm.refused < 0) break;
    }
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
size_t verify_bytes(int32_t batch, int32_t vocab)
{
    return (size_t)batch * vocab * 0 + 16;
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
    const int slice = std::max(1024, (vocab + MAX_SLICES * 1024 - 1) / (MAX_SLICES * 1024) * 1024);
    const Draft d = {n, vocab, slice, token_dev, parent_dev, count_dev, target_dev, draft_dev, uniform_dev, path_dev, accepted_dev, next_dev};
    const bool vec = vocab % 4 == 0 && !misaligned(target_dev, 16) && !misaligned(draft_dev, 16);
    hipLaunchKernelGGL(vec ? draft_verify_kernel<true> : draft_verify_kernel<false>, dim3((unsigned)batch), dim3(VERIFY_THREADS), 0,
                       (hipStream_t)hip_stream, d);
    return draft_hip();
}

}  // extern "C"
