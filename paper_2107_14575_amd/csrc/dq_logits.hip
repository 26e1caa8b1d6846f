// Between a model's logits and their gradient: log-probabilities of the tokens that were taken, the clipped policy loss with a KL
// term, the preference loss over pairs of sequences.
//
// With x_v = z_v / T, m = max_v z_v and s = sum_v exp((z_v - m) / T):
//     logp = (z_y - m) / T - ln s,       dL/dz_v = (scale * dL/dlogp / T) * ([v = y] - exp((z_v - m) / T) / s).
// A row's maximum and sum are taken in one pass (a running maximum, the sum rescaled when it grows); differences are taken before
// the scale, so that logits at their type's lowest value do not overflow, and a row's NaN or +inf gives NaN, -inf a probability of 0.
// Everything is binary32 from the loaded logit to the one rounding of the stored gradient; what is added over rows is binary64.
//
// A logit takes about 13 instructions for sum and gradient (bfloat16: unpack, maximum, difference, scale, exponential, addition; unpack, difference,
// scale, exponential, product, half a conversion), a byte read or written a quarter of that, so the memory binds all but small calls, and the
// kernels' aim is to move each byte once, whole lines at a time:
//     k_token_logprob   reads once                  8192 x 32768 bfloat16       81 us         6.6 TB/s   vector ALU issuing 67 % of the time
//     k_token_gradient  reads and writes once       2048 x 32768 bfloat16       44 us         6.1 TB/s                      26 % (at 3637 x 100003)
//     k_policy_fused    reads and writes once       4096 x 131072 bfloat16     353 to 364 us 5.9 to 6.1 TB/s               50 %
// (a copy of 2 GiB by torch: 4.9 TB/s).  The preference loss has to know all rows of a pair before the first gradient and reads twice.  Small calls are
// their launches: 2.8 us each on the host, beside 1.6 to 3.3 for a call's arguments.
#include <cmath>
#include <limits>
#include <type_traits>

#include "dq_internal.h"
#include "dq_logits.h"
#include "dq_vectors.h"

namespace {

constexpr int THREADS = 256;
constexpr int64_t MAX_STRIDE = INT64_C(1) << 38; // of elements: 2^24 rows' offsets fit 64 bits

// ---- maximum and sum -------------------------------------------------------------------------------------------------------
// the pair (maximum, sum of exp2((x - maximum) * c)) of a part of a row
struct row_sum {
    float top, sum;
};
// what is subtracted: the maximum, but where that is -inf, so that exp2 of -inf - 0 gives the 0 which such elements add
__device__ __forceinline__ float subtracted(float top) { return top == -INFINITY ? 0.0f : top; }
__device__ __forceinline__ float scaled_exp(float x, float top, float c) { return __builtin_amdgcn_exp2f((x - top) * c); }

template <int N>
__device__ __forceinline__ float largest(const float (&x)[N])
{
    float m = fmaxf(x[0], x[1]);
    for (int k = 2; k < N; k += 2) m = fmaxf(fmaxf(m, x[k]), x[k + 1]);
    return m;
}
// mine with N more elements: one rescaling for all of them, their sum as a tree
template <int N>
__device__ __forceinline__ void take(row_sum& mine, const float (&x)[N], float c)
{
    const float top = fmaxf(mine.top, largest(x)), ref = subtracted(top);
    float e[N];
    for (int k = 0; k < N; ++k) e[k] = scaled_exp(x[k], ref, c);
    for (int n = N / 2; n > 0; n /= 2)
        for (int k = 0; k < n; ++k) e[k] += e[k + n];
    mine.sum = mine.sum * scaled_exp(mine.top, ref, c) + e[0];
    mine.top = top;
}
__device__ __forceinline__ void take_one(row_sum& mine, float x, float c)
{
    const float top = fmaxf(mine.top, x), ref = subtracted(top);
    mine.sum = mine.sum * scaled_exp(mine.top, ref, c) + scaled_exp(x, ref, c);
    mine.top = top;
}

// a value of all LANES (16, 32 or 64) lanes, in every one of them; the order is fixed
template <int LANES, typename F>
__device__ __forceinline__ float lanes_all(float x, F&& op)
{
    const auto moved = [](float v, auto control) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(control)::value, 0xF, 0xF, true));
    };
    x = op(x, moved(x, std::integral_constant<int, 0xB1>{}));  // quad_perm [1, 0, 3, 2]
    x = op(x, moved(x, std::integral_constant<int, 0x4E>{}));  // quad_perm [2, 3, 0, 1]
    x = op(x, moved(x, std::integral_constant<int, 0x124>{})); // row_ror 4
    x = op(x, moved(x, std::integral_constant<int, 0x128>{})); // row_ror 8
    if constexpr (LANES == 16) return x;
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    if constexpr (LANES == 32) return x;
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return op(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}
template <int LANES>
__device__ __forceinline__ row_sum lanes_joined(row_sum mine, float c)
{
    const float top = lanes_all<LANES>(mine.top, [](float a, float b) { return fmaxf(a, b); });
    const float part = mine.sum * scaled_exp(mine.top, subtracted(top), c);
    return { top, lanes_all<LANES>(part, [](float a, float b) { return a + b; }) };
}
// all TH threads' parts; 16 lanes or a wavefront have a row of their own
template <int TH>
__device__ __forceinline__ row_sum joined(row_sum mine, float c)
{
    if constexpr (TH <= 64) return lanes_joined<TH>(mine, c);
    mine = lanes_joined<64>(mine, c);
    __shared__ row_sum parts[TH < 64 ? 1 : TH / 64];
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x / 64] = mine;
    __syncthreads();
    const int lane = threadIdx.x & 63;
    return lanes_joined<64>(lane < TH / 64 ? parts[lane] : row_sum{ -INFINITY, 0.0f }, c);
}

// Workgroups beyond 2^20 are counted in the grid's second dimension: a dimension's threads have to fit 32 bits.
constexpr int64_t GRID_X = 1 << 20;
__device__ __forceinline__ int64_t workgroup() { return static_cast<int64_t>(blockIdx.y) * GRID_X + blockIdx.x; }

// TH threads for each row: a workgroup of 256 takes several rows where that is 16, 32 or 64, otherwise one.  Small rows share a wavefront, so that its
// instructions for a row's scalars and its reductions serve several (loss and gradient of 65536 rows of 500 bfloat16 60 -> 34 us).
template <int TH>
constexpr int WORKGROUP = TH <= 64 ? THREADS : TH;
template <int TH>
constexpr int ROWS_AT_ONCE = WORKGROUP<TH> / TH;
// this thread's row among its workgroup's; a wavefront's own if TH = 64
template <int TH>
__device__ __forceinline__ int row_in_workgroup()
{
    if constexpr (TH == 64) return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / 64));
    return threadIdx.x / TH;
}
template <int TH>
constexpr int BEHIND = TH == 16 ? 8 : TH / 2 < 32 ? TH / 2 : 32; // the thread from which on a row's last elements are taken

// The last of n workgroups to arrive at a counter, asked by one wavefront whose lane 0 has stored what the others are to see; the counter goes back to zero.
// What is handed over is stored and loaded at device scope (an XCD's cache is not another's: such stores go through it, such loads pass it by), and the store
// is complete before the counter moves.  A release of everything the workgroup has written would write the XCD's whole cache back, gradients and all: 64 rows of
// 131072 logits 20 -> 30 us.  The counters are the library's own, one set on each GPU, so only calls on the default stream use them, which run one after the
// other whatever thread makes them and cannot be captured.
constexpr uint32_t GROUP = 64; // workgroups that arrive at one counter: 25 ns each
struct __align__(256) arrival_counter {
    uint32_t n;
};
__device__ arrival_counter arrived[DQ_ARRIVE_WORKGROUPS], groups_arrived;
template <typename T>
__device__ __forceinline__ void store_shared(T* at, T v)
{
    __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T load_shared(const T* at)
{
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool last_to_arrive(uint32_t* counter, uint32_t n)
{
    uint32_t ticket = 0;
    if ((threadIdx.x & 63) == 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        ticket = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(ticket))) != n - 1) return false;
    if ((threadIdx.x & 63) == 0) store_shared(counter, 0u);
    asm volatile("" ::: "memory");
    return true;
}

__device__ __forceinline__ float log_probability(float of_token, const row_sum& all, double inv_t)
{
    // the difference in binary64: in binary32 it overflows for logits at both ends of the type, where its product with a small 1 / T does not
    return static_cast<float>((static_cast<double>(of_token) - static_cast<double>(all.top)) * inv_t - static_cast<double>(logf(all.sum)));
}

// adds the vectors first, first + step, ... below end of a row to `mine`.  STREAM: logits that nothing reads again; without it the last 256 MB of them stay in the
// last-level cache for the gradient (8192 x 32768 bfloat16: 93 -> 82 us alone; with the gradient of 2500 x 30000 behind them 76 -> 81).
template <bool STREAM, typename T>
__device__ __forceinline__ void take_vectors(row_sum& mine, const T* body, int first, int end, int step, float c)
{
    constexpr int AT_ONCE = 4; // in flight of a thread
    for (int at = first; at < end; at += AT_ONCE * step) {
        vec v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            for (int j = 0; j < 4; ++j) v[i][j] = MINUS_INF<T>;
            if (at + i * step < end) v[i] = load_vec<STREAM>(body + static_cast<int64_t>(at + i * step) * PER<T>);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            float x[PER<T>];
            unpack<T>(v[i], x);
            take(mine, x, c);
        }
    }
}

struct forward_args {
    dq_rows rows;
    const int64_t* tokens;
    const float* weights; // or null
    double inv_t;
    float c;
    float* logp;
    float2* softmax; // or null
    float* dlogp;    // or null: set to zero
    __device__ __forceinline__ bool counts(int64_t r, int64_t y) const { return y >= 0 && y < rows.vocab && !(weights && weights[r] == 0.0f); }
    __device__ __forceinline__ void write(int64_t r, float lp, float top, float inv_sum) const
    {
        logp[r] = lp;
        if (softmax) softmax[r] = make_float2(top, inv_sum);
        if (dlogp) dlogp[r] = 0.0f;
    }
};

// A row's maximum and sum, and the taken token's log-probability, by TH threads: write(log-probability, maximum, 1 / sum) by the first of them
template <typename T, int TH, bool STREAM, typename F>
__device__ __forceinline__ void forward_row(const forward_args& a, int64_t r, int tid, F&& write)
{
    const int64_t y = a.tokens[r];
    if (!a.counts(r, y)) {
        if (tid == 0) write(0.0f, 0.0f, 0.0f);
        return;
    }
    const T* z = static_cast<const T*>(a.rows.data) + a.rows.at(r);
    const float of_token = static_cast<float>(z[y]);
    const dq_parts<T> parts(z, a.rows.vocab);
    row_sum mine = { -INFINITY, 0.0f };
    const int end = parts.template end_of<BEHIND<TH>>(tid, a.rows.vocab);
    if (end >= 0) take_one(mine, static_cast<float>(z[end]), a.c);
    take_vectors<STREAM>(mine, z + parts.head, tid, parts.vecs, TH, a.c);
    const row_sum all = joined<TH>(mine, a.c);
    if (tid == 0) write(log_probability(of_token, all, a.inv_t), all.top, 1.0f / all.sum);
}
template <typename T, int TH, bool STREAM>
__global__ __launch_bounds__(WORKGROUP<TH>) void k_token_logprob(forward_args a)
{
    const int64_t r = workgroup() * ROWS_AT_ONCE<TH> + row_in_workgroup<TH>();
    if (r >= a.rows.count) return;
    forward_row<T, TH, STREAM>(a, r, threadIdx.x & (TH - 1), [&](float lp, float top, float inv_sum) { a.write(r, lp, top, inv_sum); });
}

// Few long rows are cut into slices, a workgroup each, so that more than `count` CUs work: one row of 131072 bfloat16 logits forward 9.8 us by one workgroup,
// 5.4 in 16 slices.  What a slice finds, and the taken token's logit, are kept in the workspace.
constexpr int MOST_SLICES = 64; // one lane for each in the join
struct row_slices {
    uint64_t* found; // [rows][slices]: a row_sum
    float* of_token; // [rows]
    int slices, vecs; // of a row, of a slice
};
__device__ __forceinline__ row_sum slices_joined(const row_slices& s, int64_t r, float c)
{
    const int lane = threadIdx.x & 63;
    return lanes_joined<64>(lane < s.slices ? __builtin_bit_cast(row_sum, load_shared(s.found + r * s.slices + lane)) : row_sum{ -INFINITY, 0.0f }, c);
}
template <typename T>
__global__ __launch_bounds__(THREADS) void k_row_slices(forward_args a, row_slices s, bool arrive)
{
    const int64_t r = blockIdx.y;
    const int slice = blockIdx.x;
    const int64_t y = a.tokens[r];
    if (!a.counts(r, y)) {
        if (arrive && slice == 0 && threadIdx.x == 0) a.write(r, 0.0f, 0.0f, 0.0f);
        return;
    }
    const T* z = static_cast<const T*>(a.rows.data) + a.rows.at(r);
    const dq_parts<T> parts(z, a.rows.vocab);
    row_sum mine = { -INFINITY, 0.0f };
    const int end = slice == 0 ? parts.end_of(threadIdx.x, a.rows.vocab) : -1;
    if (end >= 0) take_one(mine, static_cast<float>(z[end]), a.c);
    take_vectors<false>(mine, z + parts.head, slice * s.vecs + static_cast<int>(threadIdx.x), min((slice + 1) * s.vecs, parts.vecs), THREADS, a.c);
    mine = joined<THREADS>(mine, a.c);
    if (threadIdx.x == 0) {
        store_shared(s.found + r * s.slices + slice, __builtin_bit_cast(uint64_t, mine));
        if (slice == 0) s.of_token[r] = static_cast<float>(z[y]);
    }
    if (!arrive || threadIdx.x >= 64 || !last_to_arrive(&arrived[r].n, static_cast<uint32_t>(s.slices))) return;
    const row_sum all = slices_joined(s, r, a.c);
    if (threadIdx.x == 0) a.write(r, log_probability(static_cast<float>(z[y]), all, a.inv_t), all.top, 1.0f / all.sum);
}
// the join by itself, a wavefront a row
__global__ __launch_bounds__(THREADS) void k_join_slices(forward_args a, row_slices s)
{
    const int64_t r = static_cast<int64_t>(blockIdx.x) * (THREADS / 64) + row_in_workgroup<64>();
    if (r >= a.rows.count) return;
    const bool counts = a.counts(r, a.tokens[r]);
    const row_sum all = counts ? slices_joined(s, r, a.c) : row_sum{ 0.0f, 1.0f };
    if ((threadIdx.x & 63) == 0) a.write(r, counts ? log_probability(s.of_token[r], all, a.inv_t) : 0.0f, all.top, counts ? 1.0f / all.sum : 0.0f);
}

// The logits' gradient from a row's maximum, inverse sum and dL/dlogp: every wavefront NV * 64 vectors of one row.  A row that does not count, or that the
// loss does not depend on, gets zeros and is not read.  Four vectors of a lane, 4 KB of a wavefront: rows need no workgroup of their own here, and as many
// workgroups as the row has slices keep all CUs busy whatever the sizes.
template <typename T, int NV>
__global__ __launch_bounds__(THREADS) void k_token_gradient(dq_rows rows, dq_rows out, uint32_t slices, const int64_t* __restrict__ tokens,
                                                            const float2* __restrict__ softmax, const float* __restrict__ dlogp, float scale, float c)
{
    const int lane = threadIdx.x & 63;
    const int64_t wave = workgroup() * (THREADS / 64) + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / 64));
    const int64_t r = wave / slices;
    if (r >= rows.count) return;
    const int slice = static_cast<int>(wave - r * slices);
    const int64_t y = tokens[r];
    const bool counts = y >= 0 && y < rows.vocab;
    const float d = counts ? dlogp[r] * scale : 0.0f;
    const T* z = static_cast<const T*>(rows.data) + rows.at(r);
    T* g = static_cast<T*>(const_cast<void*>(out.data)) + out.at(r);
    const dq_parts<T> parts(z, rows.vocab);
    const int first = slice * NV * 64 + lane, end = slice == 0 ? parts.end_of(lane, rows.vocab) : -1;
    if (d == 0.0f) {
        const vec zero = { 0, 0, 0, 0 };
        for (int i = 0; i < NV; ++i)
            if (first + i * 64 < parts.vecs) store_vec(g + parts.head + static_cast<int64_t>(first + i * 64) * PER<T>, zero);
        if (end >= 0) g[end] = static_cast<T>(0.0f);
        return;
    }
    vec v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (first + i * 64 < parts.vecs) v[i] = load_vec<true>(z + parts.head + static_cast<int64_t>(first + i * 64) * PER<T>);
    const float of_end = end >= 0 ? static_cast<float>(z[end]) : 0.0f;
    const float of_token = static_cast<float>(z[y]);
    const float2 ms = softmax[r];
    const float k = -d * ms.y;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (first + i * 64 < parts.vecs) {
            float x[PER<T>];
            unpack<T>(v[i], x);
            for (int j = 0; j < PER<T>; ++j) x[j] = scaled_exp(x[j], ms.x, c) * k;
            store_vec(g + parts.head + static_cast<int64_t>(first + i * 64) * PER<T>, pack<T>(x));
        }
    if (end >= 0) g[end] = static_cast<T>(scaled_exp(of_end, ms.x, c) * k);
    // the token's own element again, by the lane that has just written it
    const int in_body = static_cast<int>(y) - parts.head;
    const int owner = in_body >= 0 && in_body < parts.vecs * PER<T> ? in_body / PER<T> - slice * NV * 64 : -1;
    if (end == y || (owner >= 0 && owner < NV * 64 && (owner & 63) == lane)) g[y] = static_cast<T>(scaled_exp(of_token, ms.x, c) * k + d);
}

// The same for small rows: 16 lanes and NV vectors of each for one (65536 rows of 100 bfloat16 12.4 -> 9.1 us; of 500 binary32, which are 125 vectors,
// 49 us by wavefronts and 88 here: too little of a line at a time).
template <typename T, int NV>
__global__ __launch_bounds__(THREADS) void k_small_gradient(dq_rows rows, dq_rows out, const int64_t* __restrict__ tokens, const float2* __restrict__ softmax,
                                                            const float* __restrict__ dlogp, float scale, float c)
{
    constexpr int TH = 16;
    const int64_t r = workgroup() * ROWS_AT_ONCE<TH> + row_in_workgroup<TH>();
    if (r >= rows.count) return;
    const int tid = threadIdx.x & (TH - 1);
    const int64_t y = tokens[r];
    const bool counts = y >= 0 && y < rows.vocab;
    const float d = counts ? dlogp[r] * scale : 0.0f;
    const T* z = static_cast<const T*>(rows.data) + rows.at(r);
    T* g = static_cast<T*>(const_cast<void*>(out.data)) + out.at(r);
    const dq_parts<T> parts(z, rows.vocab);
    const int end = parts.template end_of<BEHIND<TH>>(tid, rows.vocab);
    const bool any = d != 0.0f; // NaN too
    vec v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (any && i * TH + tid < parts.vecs) v[i] = load_vec<true>(z + parts.head + (i * TH + tid) * PER<T>);
    const float of_end = any && end >= 0 ? static_cast<float>(z[end]) : 0.0f;
    const float of_token = any ? static_cast<float>(z[y]) : 0.0f;
    const float2 ms = any ? softmax[r] : make_float2(0.0f, 0.0f);
    const float k = -d * ms.y;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * TH + tid < parts.vecs) {
            float x[PER<T>];
            unpack<T>(v[i], x);
            for (int j = 0; j < PER<T>; ++j) x[j] = any ? scaled_exp(x[j], ms.x, c) * k : 0.0f;
            store_vec<false>(g + parts.head + (i * TH + tid) * PER<T>, pack<T>(x));
        }
    if (end >= 0) g[end] = static_cast<T>(any ? scaled_exp(of_end, ms.x, c) * k : 0.0f);
    const int in_body = static_cast<int>(y) - parts.head;
    const bool owner = in_body >= 0 && in_body < parts.vecs * PER<T> ? (in_body / PER<T> & (TH - 1)) == tid : end == y;
    if (any && owner) g[y] = static_cast<T>(scaled_exp(of_token, ms.x, c) * k + d);
}

struct policy_args {
    const float *old_logp, *ref_logp, *advantages, *weights;
    float low, high, beta; // 1 - clip_low, 1 + clip_high
};

// a row's scalars, loaded with its first vectors
struct policy_scalars {
    float w, a, old_logp, ref_logp;
    __device__ __forceinline__ policy_scalars(const policy_args& p, int64_t r)
        : w(p.weights[r]), a(p.advantages[r]), old_logp(p.old_logp[r]), ref_logp(p.ref_logp ? p.ref_logp[r] : 0.0f)
    {
    }
};
// One row's terms of the policy loss, and the loss's derivative by its log-probability.
__device__ __forceinline__ float4 policy_row(const policy_args& p, const policy_scalars& s, float logp, float& d)
{
    const float w = s.w, a = s.a;
    const float change = logp - s.old_logp, ratio = expf(change);
    float plain = ratio * a;
    const float clipped = fminf(fmaxf(ratio, p.low), p.high) * a;
    if (ratio == INFINITY) { // the product may be a number of binary32 all the same, as 0 is for an advantage of 0
        const float half = expf(0.5f * change);
        plain = half * a * half;
    }
    const bool active = !(plain > clipped); // also where one is NaN, which then shows
    const float term = active ? -plain : -clipped;
    float kl = 0.0f, penalty = 0.0f;
    d = active ? -plain : 0.0f;
    if (p.ref_logp) {
        const float u = s.ref_logp - logp, e = expm1f(u);
        kl = e == INFINITY ? e : e - u; // of a token of probability 0 infinite, not NaN
        if (p.beta != 0.0f) { // a divergence that is only looked at may be infinite
            penalty = p.beta * kl;
            d -= p.beta * e;
        }
    }
    d *= w;
    return make_float4(w * (term + penalty), w * term, w * kl, active ? 0.0f : w);
}

// a workgroup's sums of the four terms, in binary64
struct term_sums {
    double of[4];
    __device__ __forceinline__ void store(term_sums* at) const
    {
        for (int k = 0; k < 4; ++k) store_shared(at->of + k, of[k]);
    }
    __device__ __forceinline__ void add(const float4& t)
    {
        of[0] += t.x;
        of[1] += t.y;
        of[2] += t.z;
        of[3] += t.w;
    }
};

// Loss terms and gradient of a row in one pass: its vectors stay in registers (NV of each of TH threads) between the sum and the gradient, so that the
// logits are read once.  REST: a row of more vectors than that; IN_LDS more of each thread are kept in LDS (each thread its own, so that there is nothing to
// wait for), and what is beyond those is read again, behind the 256 MB of the last-level cache.
// One row's loads, sums and stores follow one another, so it is several rows on a CU that keep the memory busy: as many threads a row as it needs for some
// vectors each and no more (the choice, with both sides measured, is policy_gradient's).  LDS: 2048 x 140000 binary32 447 -> 395 us, 1024 x 200000 347 -> 301.
constexpr int IN_LDS = 9; // 144 KB of 1024 threads
template <typename T, int TH, int NV, bool REST>
__device__ __forceinline__ float4 policy_of_row(int64_t r, int tid, const dq_rows& rows, const dq_rows& out, const int64_t* __restrict__ tokens, const policy_args& p,
                                                double inv_t, float c, float scale, float* __restrict__ logp)
{
    const int64_t y = tokens[r];
    const policy_scalars scalars(p, r);
    const bool counts = y >= 0 && y < rows.vocab && scalars.w != 0.0f;
    T* g = static_cast<T*>(const_cast<void*>(out.data)) + out.at(r);
    const T* z = static_cast<const T*>(rows.data) + rows.at(r);
    const dq_parts<T> parts(z, rows.vocab);
    const int end = parts.template end_of<BEHIND<TH>>(tid, rows.vocab);
    const T* body = z + parts.head;
    T* gbody = g + parts.head;
    const auto zeros = [&] {
        const vec zero = { 0, 0, 0, 0 };
        for (int k = tid; k < parts.vecs; k += TH) store_vec(gbody + static_cast<int64_t>(k) * PER<T>, zero);
        if (end >= 0) g[end] = static_cast<T>(0.0f);
    };
    if (!counts) {
        if (tid == 0) logp[r] = 0.0f;
        zeros();
        return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    row_sum mine = { -INFINITY, 0.0f };
    vec* held = nullptr; // this thread's in LDS, TH apart
    if constexpr (REST) {
        __shared__ vec in_lds[IN_LDS * TH];
        held = in_lds + tid;
        take_vectors<false>(mine, body, TH * (NV + IN_LDS) + tid, parts.vecs, TH, c);
        constexpr int AT_ONCE = 3;
        static_assert(IN_LDS % AT_ONCE == 0, "whole rounds");
#pragma unroll 1
        for (int i = 0; i < IN_LDS; i += AT_ONCE) {
            vec v[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int k = TH * (NV + i + j) + tid;
                for (int w = 0; w < 4; ++w) v[j][w] = MINUS_INF<T>;
                if (k < parts.vecs) v[j] = load_vec<true>(body + static_cast<int64_t>(k) * PER<T>);
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                float x[PER<T>];
                unpack<T>(v[j], x);
                take(mine, x, c);
                held[(i + j) * TH] = v[j];
            }
        }
    }
    vec v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int k = i * TH + tid;
        for (int j = 0; j < 4; ++j) v[i][j] = MINUS_INF<T>;
        if (k < parts.vecs) v[i] = load_vec<true>(body + static_cast<int64_t>(k) * PER<T>);
    }
    const float of_end = end >= 0 ? static_cast<float>(z[end]) : -INFINITY;
    const float of_token = static_cast<float>(z[y]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * TH < parts.vecs) {
            float x[PER<T>];
            unpack<T>(v[i], x);
            take(mine, x, c);
        }
    }
    take_one(mine, of_end, c);
    const row_sum all = joined<TH>(mine, c);
    // the row's scalars, in every thread: cheaper than a second barrier
    const float lp = log_probability(of_token, all, inv_t);
    float d = 0.0f;
    const float4 terms = policy_row(p, scalars, lp, d);
    if (tid == 0) logp[r] = lp;
    d *= scale;
    if (d == 0.0f) { // the clip stops it
        zeros();
        return terms;
    }
    const float k = -d / all.sum;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * TH + tid < parts.vecs) {
            float x[PER<T>];
            unpack<T>(v[i], x);
            for (int j = 0; j < PER<T>; ++j) x[j] = scaled_exp(x[j], all.top, c) * k;
            store_vec<(TH > 16)>(gbody + static_cast<int64_t>(i * TH + tid) * PER<T>, pack<T>(x));
        }
    }
    if constexpr (REST) {
        const auto write = [&](int at, const vec& v) {
            float x[PER<T>];
            unpack<T>(v, x);
            for (int j = 0; j < PER<T>; ++j) x[j] = scaled_exp(x[j], all.top, c) * k;
            store_vec(gbody + static_cast<int64_t>(at) * PER<T>, pack<T>(x));
        };
#pragma unroll 3
        for (int i = 0; i < IN_LDS; ++i)
            if (TH * (NV + i) + tid < parts.vecs) write(TH * (NV + i) + tid, held[i * TH]);
        constexpr int AT_ONCE = 4;
        for (int at = TH * (NV + IN_LDS) + tid; at < parts.vecs; at += AT_ONCE * TH) {
            vec v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                if (at + i * TH < parts.vecs) v[i] = load_vec<true>(body + static_cast<int64_t>(at + i * TH) * PER<T>);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                if (at + i * TH < parts.vecs) write(at + i * TH, v[i]);
        }
    }
    if (end >= 0) g[end] = static_cast<T>(scaled_exp(of_end, all.top, c) * k);
    // the token's own element again, by the thread that has just written it
    const int in_body = static_cast<int>(y) - parts.head;
    const bool owner = in_body >= 0 && in_body < parts.vecs * PER<T> ? (in_body / PER<T> & (TH - 1)) == tid : end == y;
    if (owner) g[y] = static_cast<T>(scaled_exp(of_token, all.top, c) * k + d);
    return terms;
}

// The sum of n workgroups' sums in one wavefront, 16 lanes for each of the four: in lane k < 4, and by symmetry in every fourth lane from there
__device__ __forceinline__ double sum_of(const term_sums* sums, uint32_t n)
{
    const uint32_t lane = threadIdx.x & 63;
    double mine = 0.0;
#pragma unroll 4
    for (uint32_t at = lane; at < 4 * n; at += 64) mine += load_shared(sums->of + at);
    for (int off = 4; off < 64; off *= 2) mine += __shfl_xor(mine, off, 64);
    return mine;
}
// The loss by the last workgroups to arrive: of GROUP of them, which adds their sums, then of the groups.  One wavefront of each workgroup asks, its lane 0 having
// stored sums[me]; behind the n sums there is room for those of the groups.  In the order of a fixed tree.
constexpr uint32_t MOST_ARRIVING = GROUP * DQ_ARRIVE_WORKGROUPS;
__device__ __forceinline__ void sum_by_last(term_sums* sums, uint32_t me, uint32_t n, double scale, float* __restrict__ loss)
{
    const uint32_t lane = threadIdx.x & 63, group = me / GROUP, groups = (n + GROUP - 1) / GROUP, in_group = min(GROUP, n - group * GROUP);
    if (!last_to_arrive(&arrived[group].n, in_group)) return;
    double mine = sum_of(sums + group * GROUP, in_group);
    if (groups > 1) {
        if (lane < 4) store_shared(sums[n + group].of + lane, mine);
        if (!last_to_arrive(&groups_arrived.n, groups)) return;
        mine = sum_of(sums + n, groups);
    }
    if (lane < 4) loss[lane] = static_cast<float>(mine * scale);
}

// What is left to add are as many sums as workgroups, which the last of them do with `loss`; then there is no second launch.
template <typename T, int TH, int NV, bool REST>
__global__ __launch_bounds__(WORKGROUP<TH>) void k_policy_fused(dq_rows rows, dq_rows out, const int64_t* __restrict__ tokens, policy_args p, double inv_t, float c,
                                                                float scale, float* __restrict__ logp, term_sums* sums, float* loss)
{
    constexpr int AT_ONCE = ROWS_AT_ONCE<TH>;
    const int which = AT_ONCE > 1 ? row_in_workgroup<TH>() : 0, tid = threadIdx.x & (TH - 1);
    const int64_t me = workgroup(), r = me * AT_ONCE + which;
    if (AT_ONCE == 1 && r >= rows.count) return;
    float4 t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (r < rows.count) t = policy_of_row<T, TH, NV, REST>(r, tid, rows, out, tokens, p, inv_t, c, scale, logp);
    term_sums mine = { { t.x, t.y, t.z, t.w } };
    if constexpr (AT_ONCE > 1) {
        __shared__ float4 of_row[AT_ONCE];
        if (tid == 0) of_row[which] = t;
        __syncthreads();
        if (me * AT_ONCE >= rows.count) return;
        for (int w = 1; w < AT_ONCE; ++w) mine.add(of_row[w]); // thread 0 has the first row
    }
    if (threadIdx.x == 0) mine.store(sums + me);
    if (loss && threadIdx.x < 64) sum_by_last(sums, static_cast<uint32_t>(me), gridDim.x, 1.0, loss);
}

// Few long rows: every slice's workgroup joins what k_row_slices found, works out the row's scalars and writes the gradient of its slice.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_policy_slices(dq_rows rows, dq_rows out, const int64_t* __restrict__ tokens, policy_args p, double inv_t, float c,
                                                           float scale, float* __restrict__ logp, term_sums* sums, float* loss, row_slices s)
{
    constexpr int AT_ONCE = 4;
    const int64_t r = blockIdx.y;
    const int slice = blockIdx.x;
    const int64_t y = tokens[r];
    const policy_scalars scalars(p, r);
    const bool counts = y >= 0 && y < rows.vocab && scalars.w != 0.0f;
    T* g = static_cast<T*>(const_cast<void*>(out.data)) + out.at(r);
    const T* z = static_cast<const T*>(rows.data) + rows.at(r);
    const dq_parts<T> parts(z, rows.vocab);
    const int end = slice == 0 ? parts.end_of(threadIdx.x, rows.vocab) : -1, last = min((slice + 1) * s.vecs, parts.vecs);
    float4 terms = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float d = 0.0f, k = 0.0f, lp = 0.0f, top = 0.0f, of_token = 0.0f;
    if (counts) {
        const row_sum all = slices_joined(s, r, c);
        of_token = s.of_token[r];
        lp = log_probability(of_token, all, inv_t);
        terms = policy_row(p, scalars, lp, d);
        d *= scale;
        k = -d / all.sum;
        top = all.top;
    }
    const bool any = d != 0.0f; // NaN too
    const float of_end = any && end >= 0 ? static_cast<float>(z[end]) : 0.0f;
    for (int at = slice * s.vecs + static_cast<int>(threadIdx.x); at < last; at += AT_ONCE * THREADS) {
        vec v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (any && at + i * THREADS < last) v[i] = load_vec<true>(z + parts.head + static_cast<int64_t>(at + i * THREADS) * PER<T>);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (at + i * THREADS < last) {
                float x[PER<T>];
                unpack<T>(v[i], x);
                for (int j = 0; j < PER<T>; ++j) x[j] = any ? scaled_exp(x[j], top, c) * k : 0.0f;
                store_vec(g + parts.head + static_cast<int64_t>(at + i * THREADS) * PER<T>, pack<T>(x));
            }
    }
    if (end >= 0) g[end] = static_cast<T>(any ? scaled_exp(of_end, top, c) * k : 0.0f);
    // the token's own element again, by the thread that has just written it
    const int in_body = static_cast<int>(y) - parts.head, vector = in_body / PER<T>;
    const bool owner = in_body >= 0 && in_body < parts.vecs * PER<T> ? vector >= slice * s.vecs && vector < last && (vector - slice * s.vecs) % THREADS == static_cast<int>(threadIdx.x)
                                                                     : end == y;
    if (any && owner) g[y] = static_cast<T>(scaled_exp(of_token, top, c) * k + d);
    if (slice == 0 && threadIdx.x == 0) {
        logp[r] = lp;
        term_sums{ { terms.x, terms.y, terms.z, terms.w } }.store(sums + r);
    }
    // the rows' sums are those of their first slices
    if (loss && slice == 0 && threadIdx.x < 64) sum_by_last(sums, blockIdx.y, gridDim.y, 1.0, loss);
}

// the terms of the loss alone, THREADS rows a workgroup
__global__ __launch_bounds__(THREADS) void k_policy_rows(policy_args p, int64_t count, int64_t vocab, const int64_t* __restrict__ tokens,
                                                         const float* __restrict__ logp, term_sums* __restrict__ sums)
{
    __shared__ double parts[4][THREADS];
    term_sums mine = { { 0.0, 0.0, 0.0, 0.0 } };
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; r < count; r += static_cast<int64_t>(gridDim.x) * THREADS)
        if (tokens[r] >= 0 && tokens[r] < vocab && p.weights[r] != 0.0f) {
            float d;
            mine.add(policy_row(p, policy_scalars(p, r), logp[r], d));
        }
    for (int k = 0; k < 4; ++k) parts[k][threadIdx.x] = mine.of[k];
    __syncthreads();
    for (int n = THREADS / 2; n > 0; n /= 2) {
        if (threadIdx.x < n)
            for (int k = 0; k < 4; ++k) parts[k][threadIdx.x] += parts[k][threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x < 4) sums[blockIdx.x].of[threadIdx.x] = parts[threadIdx.x][0];
}

// The sums' sums, in binary64 and in a fixed order: four threads for each of 256 of them at a time.  Workgroup b of a grid adds those in its share of `each` into
// part[b]; a grid of one, of all of them, scales the result into loss[0..3].
constexpr int SUM_THREADS = 1024;
__global__ __launch_bounds__(SUM_THREADS) void k_sum_terms(const term_sums* __restrict__ sums, int64_t count, int64_t each, double scale, term_sums* __restrict__ part,
                                                           float* __restrict__ loss)
{
    __shared__ double parts[SUM_THREADS];
    const double* of = sums->of;
    const int64_t first = 4 * each * blockIdx.x, end = min(first + 4 * each, 4 * count);
    double mine[4] = { 0.0, 0.0, 0.0, 0.0 };
    for (int64_t at = first + threadIdx.x; at < end; at += 4 * SUM_THREADS)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k * SUM_THREADS < end) mine[k] += of[at + k * SUM_THREADS];
    parts[threadIdx.x] = (mine[0] + mine[1]) + (mine[2] + mine[3]);
    __syncthreads();
    for (int n = SUM_THREADS / 2; n >= 4; n /= 2) {
        if (threadIdx.x < n) parts[threadIdx.x] += parts[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x < 4) {
        if (loss)
            loss[threadIdx.x] = static_cast<float>(parts[threadIdx.x] * scale);
        else
            part[blockIdx.x].of[threadIdx.x] = parts[threadIdx.x];
    }
}

struct preference_args {
    const int64_t* seq_start; // [2 * pairs + 1]
    const float* ref_logp;    // [2 * pairs] or null
    int64_t pairs, rows, vocab;
    float beta, smoothing;
    bool average;
};

// A pair's numbers from its sequences' sums and counts of log-probabilities.
struct pair_result {
    double total[2], reward[2], loss, h;
    float d[2]; // dL/dlogp of a token of each sequence
};
__device__ __forceinline__ pair_result pair_of(const preference_args& p, const double (&sum)[2], const int (&counted)[2], const double (&ref)[2])
{
    pair_result r;
    double by[2];
    for (int k = 0; k < 2; ++k) {
        by[k] = p.average && counted[k] > 1 ? static_cast<double>(counted[k]) : 1.0;
        r.total[k] = sum[k] / by[k];
        r.reward[k] = static_cast<double>(p.beta) * (r.total[k] - ref[k]);
    }
    const double h = r.reward[0] - r.reward[1], eps = p.smoothing;
    const double e = exp(-fabs(h)), rest = log1p(e); // -ln sigma(h) = rest + max(-h, 0)
    // a sequence of probability 0 makes h infinite: the term whose factor is 0 is 0 then, not 0 times infinity
    const double loss = (eps < 1.0 ? (1.0 - eps) * (rest + fmax(-h, 0.0)) : 0.0) + (eps > 0.0 ? eps * (rest + fmax(h, 0.0)) : 0.0);
    const double sigma = (h > 0.0 ? e : 1.0) / (1.0 + e); // of -h
    const double g = static_cast<double>(p.beta) * ((1.0 - eps) * sigma - eps * (1.0 - sigma)) / static_cast<double>(p.pairs);
    r.h = h;
    r.loss = h == h ? loss : h;
    for (int k = 0; k < 2; ++k) r.d[k] = static_cast<float>((h == h ? (k ? g : -g) : h) / by[k]);
    return r;
}
struct pair_rows {
    int64_t of[2], first[2], end[2]; // sequences, their rows
    double ref[2];
    __device__ __forceinline__ pair_rows(const preference_args& p, int64_t pair)
    {
        for (int k = 0; k < 2; ++k) {
            of[k] = pair + k * p.pairs;
            first[k] = min(max(p.seq_start[of[k]], static_cast<int64_t>(0)), p.rows);
            end[k] = min(max(p.seq_start[of[k] + 1], static_cast<int64_t>(0)), p.rows);
            ref[k] = p.ref_logp ? p.ref_logp[of[k]] : 0.0;
        }
    }
};

// One workgroup per pair, a half of it for each sequence: the sequences' log-probabilities (binary64, fixed order), the pair's terms, and dL/dlogp of their tokens.
__global__ __launch_bounds__(THREADS) void k_preference_pairs(preference_args p, const int64_t* __restrict__ tokens, const float* __restrict__ logp,
                                                              term_sums* terms, float* __restrict__ seq_logp, float* __restrict__ dlogp, float* loss)
{
    constexpr int HALF = THREADS / 2, WAVES = THREADS / 64;
    static_assert(WAVES == 4, "two wavefronts a sequence");
    __shared__ double sums[WAVES];
    __shared__ int counts[WAVES];
    const int64_t pair = workgroup();
    if (pair >= p.pairs) return;
    const pair_rows rows(p, pair);
    const int wave = threadIdx.x / 64, mine = threadIdx.x / HALF, tid = threadIdx.x % HALF; // which sequence: 0 the preferred one
    const int64_t first = mine ? rows.first[1] : rows.first[0], end = mine ? rows.end[1] : rows.end[0];
    double sum = 0.0;
    int n = 0;
#pragma unroll 4
    for (int64_t r = first + tid; r < end; r += HALF) {
        sum += logp[r]; // 0 where the token does not count
        n += tokens[r] >= 0 && tokens[r] < p.vocab;
    }
    for (int off = 32; off > 0; off /= 2) {
        sum += __shfl_xor(sum, off, 64);
        n += __shfl_xor(n, off, 64);
    }
    if ((threadIdx.x & 63) == 0) {
        sums[wave] = sum;
        counts[wave] = n;
    }
    __syncthreads();
    // the pair's numbers, in every thread
    const pair_result of_pair = pair_of(p, { sums[0] + sums[1], sums[2] + sums[3] }, { counts[0] + counts[1], counts[2] + counts[3] }, rows.ref);
    const float d = mine ? of_pair.d[1] : of_pair.d[0];
    for (int64_t r = first + tid; r < end; r += HALF) dlogp[r] = d;
    if (threadIdx.x >= 64) return;
    if (threadIdx.x == 0) {
        term_sums{ { of_pair.loss, of_pair.h > 0.0 ? 1.0 : 0.0, of_pair.reward[0], of_pair.reward[1] } }.store(terms + pair);
        for (int k = 0; k < 2; ++k) seq_logp[rows.of[k]] = static_cast<float>(of_pair.total[k]);
    }
    if (loss) sum_by_last(terms, static_cast<uint32_t>(pair), gridDim.x, 1.0 / static_cast<double>(p.pairs), loss);
}

// Few rows and few pairs: the forward pass's last workgroup to arrive does the pairs as well, a wavefront each, and there is one launch for two.  One pair of
// 4 tokens 10.2 -> 7.8 us, four of 24 12.6 -> 11.2; eight of 100 13.6 -> 14.5, sixteen of 60 12.4 -> 17.4.  At the limits it is as fast or loses 1 to 2 us: four pairs
// of 64 tokens over 500 binary32 logits 10.4 -> 10.2, eight of 32 10.5 -> 12.2; rows of 2049 to 4096 vectors, which have 256 threads here and 1024 there: one pair of 10
// over 24000 bfloat16 12.1 -> 11.2, four of 16 over 30000 14.4 -> 16.0; beyond 4096 vectors two of 20 over 18000 binary32 14.8 -> 15.9.
constexpr int64_t FEW_PAIRS = 8, FEW_PAIR_ROWS = 512;
template <typename T, int TH>
__global__ __launch_bounds__(THREADS) void k_preference_few(forward_args a, preference_args p, float* __restrict__ seq_logp, float* __restrict__ dlogp, float* __restrict__ loss)
{
    constexpr int WAVES = THREADS / 64;
    static_assert(WORKGROUP<TH> == THREADS, "four wavefronts");
    const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS_AT_ONCE<TH> + row_in_workgroup<TH>();
    if (row < a.rows.count)
        forward_row<T, TH, false>(a, row, threadIdx.x & (TH - 1), [&](float lp, float top, float inv_sum) {
            store_shared(a.logp + row, lp);
            if (a.softmax) a.softmax[row] = make_float2(top, inv_sum);
        });
    __shared__ bool last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // every wavefront's log-probabilities, before the first one's arrival
    __syncthreads();
    if (threadIdx.x < 64) {
        const bool is_last = last_to_arrive(&arrived[0].n, gridDim.x);
        if (threadIdx.x == 0) last = is_last;
    }
    __syncthreads();
    if (!last) return;
    for (int64_t r = threadIdx.x; r < p.rows; r += THREADS) dlogp[r] = 0.0f; // of rows in no sequence
    __syncthreads();
    const int wave = row_in_workgroup<64>(), lane = threadIdx.x & 63;
    __shared__ term_sums of_wave[WAVES];
    term_sums mine = { { 0.0, 0.0, 0.0, 0.0 } };
    for (int64_t pair = wave; pair < p.pairs; pair += WAVES) {
        const pair_rows rows(p, pair);
        double sum[2] = { 0.0, 0.0 };
        int n[2] = { 0, 0 };
        for (int k = 0; k < 2; ++k) {
#pragma unroll 4
            for (int64_t r = rows.first[k] + lane; r < rows.end[k]; r += 64) {
                sum[k] += load_shared(a.logp + r);
                n[k] += a.tokens[r] >= 0 && a.tokens[r] < p.vocab;
            }
        }
        for (int off = 32; off > 0; off /= 2)
            for (int k = 0; k < 2; ++k) {
                sum[k] += __shfl_xor(sum[k], off, 64);
                n[k] += __shfl_xor(n[k], off, 64);
            }
        const pair_result of_pair = pair_of(p, sum, n, rows.ref);
        for (int k = 0; k < 2; ++k)
            for (int64_t r = rows.first[k] + lane; r < rows.end[k]; r += 64) dlogp[r] = of_pair.d[k];
        mine.of[0] += of_pair.loss;
        mine.of[1] += of_pair.h > 0.0 ? 1.0 : 0.0;
        mine.of[2] += of_pair.reward[0];
        mine.of[3] += of_pair.reward[1];
        if (lane < 2) seq_logp[lane ? rows.of[1] : rows.of[0]] = static_cast<float>(lane ? of_pair.total[1] : of_pair.total[0]);
    }
    if (lane == 0) of_wave[wave] = mine;
    __syncthreads();
    if (threadIdx.x < 4) {
        double all = 0.0;
        for (int w = 0; w < WAVES; ++w) all += of_wave[w].of[threadIdx.x];
        loss[threadIdx.x] = static_cast<float>(all / static_cast<double>(p.pairs));
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

// DQ_OK and the rows, or why not
int rows_of(const dq_logits_t* m, dq_rows& out)
{
    if (!m || m->batch < 0 || m->rows < 0 || m->vocab < 1 || m->vocab > INT32_MAX) return DQ_ERR_INVALID_ARG;
    if (m->dtype != DQ_F32 && m->dtype != DQ_F16 && m->dtype != DQ_BF16) return DQ_ERR_INVALID_ARG;
    if (m->rows > INT32_MAX || m->batch > INT32_MAX || (m->rows && m->batch > DQ_MAX_ROWS / m->rows)) return DQ_ERR_INVALID_ARG;
    out = { m->data_dev, m->batch * m->rows, m->rows, static_cast<int32_t>(m->vocab), m->batch_stride, m->row_stride };
    if (out.count == 0) return DQ_OK;
    if (!m->data_dev || !aligned(m->data_dev, m->dtype == DQ_F32 ? 4 : 2)) return DQ_ERR_INVALID_ARG;
    return m->row_stride >= 0 && m->batch_stride >= 0 && m->row_stride <= MAX_STRIDE && m->batch_stride <= MAX_STRIDE ? DQ_OK : DQ_ERR_INVALID_ARG;
}
// rows of size `inner`, n of them `stride` apart, do not meet
bool apart(int64_t n, int64_t stride, int64_t inner) { return n <= 1 || stride >= inner; }
int gradient_of(const dq_logits_t* m, const dq_logits_t* logits, dq_rows& out)
{
    const int rc = rows_of(m, out);
    if (rc != DQ_OK) return rc;
    if (m->dtype != logits->dtype || m->batch != logits->batch || m->rows != logits->rows || m->vocab != logits->vocab) return DQ_ERR_INVALID_ARG;
    if (out.count == 0) return DQ_OK;
    // every row is written by a workgroup of its own: batch by batch, or with the batch inside the rows
    const int64_t in_batch = (m->rows - 1) * m->row_stride + m->vocab, in_row = (m->batch - 1) * m->batch_stride + m->vocab;
    const bool outer = apart(m->rows, m->row_stride, m->vocab) && apart(m->batch, m->batch_stride, in_batch);
    const bool inner = apart(m->batch, m->batch_stride, m->vocab) && apart(m->rows, m->row_stride, in_row);
    return outer || inner ? DQ_OK : DQ_ERR_INVALID_ARG;
}
int64_t up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

float exp2_scale(double temperature) { return static_cast<float>(1.4426950408889634 / temperature); } // log2(e) / T
// The kernels' own factors have to be numbers of binary32.  A difference of two logits may pass binary32 and is -inf then, which is right where its
// exponential is 0 anyway: up to T = 3.27e36.  (Far beyond that the factor is 0, and its product with the -inf of a row's first maximum NaN.)
bool usable(double temperature, double scale)
{
    const float c = exp2_scale(temperature);
    return temperature > 0.0 && std::isfinite(temperature) && std::isfinite(scale) && std::isfinite(c) &&
           static_cast<double>(c) * std::numeric_limits<float>::max() >= 150.0 && std::isfinite(static_cast<float>(scale / temperature));
}

dim3 grid_of(int64_t workgroups)
{
    return workgroups <= GRID_X ? dim3(static_cast<unsigned>(workgroups)) : dim3(static_cast<unsigned>(GRID_X), static_cast<unsigned>((workgroups + GRID_X - 1) / GRID_X));
}


// Vectors of a row up to which 16 lanes or a wavefront take it.
constexpr int LANES_VECS = 128, WAVE_VECS = 512;

// Few long rows are sliced.  Loss and gradient of 24 and 64 rows of 131072 bfloat16 logits 16.3 -> 11.5 and 17.3 -> 13.8 us, of 24 rows of 30000 8.2 -> 10.5.  Beyond 64
// rows it goes by their length: 80 rows of 65536, 131072 and 262144 logits 11.8 -> 13.1, 17.6 -> 15.7 and 32.6 -> 23.9 us, 192 rows 13.5 -> 17.2, 23.7 -> 27.7 and
// 43.5 -> 48.7; a limit that rises with the length would gain up to a third between 65 and 128 rows.
bool sliced(int64_t rows, int64_t vecs) { return rows <= 64 && vecs >= 8192; }
int64_t slices_bytes(int64_t rows) { return up(rows * MOST_SLICES * static_cast<int64_t>(sizeof(row_sum))) + up(rows * 4); }
row_slices slices_of(int64_t rows, int64_t vecs, void* workspace)
{
    constexpr int64_t LEAST = 4 * THREADS; // 16 KB
    const int64_t each = (vecs + MOST_SLICES * LEAST - 1) / (MOST_SLICES * LEAST) * LEAST;
    char* at = static_cast<char*>(workspace);
    return { reinterpret_cast<uint64_t*>(at), reinterpret_cast<float*>(at + up(rows * MOST_SLICES * static_cast<int64_t>(sizeof(row_sum)))),
             static_cast<int>((vecs + each - 1) / each), static_cast<int>(each) };
}
// of a call whose type is not known yet: binary32 rows have the most vectors
int64_t slices_room(int64_t rows, int64_t vocab) { return sliced(rows, vocab / 4) ? slices_bytes(rows) : 0; }
int per_of(int dtype) { return dtype == DQ_F32 ? 4 : 8; }

// workspace: slices_bytes(rows), where few long rows may come
void forward(int dtype, const forward_args& a, void* workspace, hipStream_t stream)
{
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const auto launch = [&](auto kernel, int64_t workgroups, int threads) { hipLaunchKernelGGL(kernel, grid_of(workgroups), dim3(threads), 0, stream, a); };
        const int64_t vecs = a.rows.vocab / PER<T>, count = a.rows.count;
        const bool few = sliced(count, vecs);
        const row_slices s = few ? slices_of(count, vecs, workspace) : row_slices{};
        if (few && count * s.slices <= DQ_ARRIVE_WORKGROUPS) { // the forward pass alone: 8 rows 9.7 -> 7.1 us, 24 (more than arrive) 10.1 -> 11.1
            const bool arrive = stream == nullptr;
            hipLaunchKernelGGL(k_row_slices<T>, dim3(static_cast<unsigned>(s.slices), static_cast<unsigned>(count)), dim3(THREADS), 0, stream, a, s, arrive);
            if (!arrive) hipLaunchKernelGGL(k_join_slices, dim3(static_cast<unsigned>((count + 3) / 4)), dim3(THREADS), 0, stream, a, s);
            return;
        }
        const auto launch_rows = [&](auto stream_flag) {
            constexpr bool STREAM = decltype(stream_flag)::value;
            if (vecs <= LANES_VECS) // 65536 rows of 260 and 512 binary32: 15.7 and 24.9 us; a wavefront 28.3 and 31.2
                launch(k_token_logprob<T, 16, STREAM>, (count + 15) / 16, THREADS);
            else if (vecs <= WAVE_VECS)
                launch(k_token_logprob<T, 64, STREAM>, (count + 3) / 4, THREADS);
            else if (vecs <= 2048 || count >= 1024) // 1000 rows of 16384 bfloat16 9.2 us, 8192 of 30000 88; 1024 threads 11.5 and 94 (2048 of 100003: 78 and 73)
                launch(k_token_logprob<T, 256, STREAM>, count, 256);
            else // 100 rows of 30000 and 100003 bfloat16 5.2 and 9.5 us; 256 threads 6.2 and 13.8 (300 to 1000 rows of 16400: 7.1 to 11.7 and 6.0 to 9.5)
                launch(k_token_logprob<T, 1024, STREAM>, count, 1024);
        };
        if (a.softmax)
            launch_rows(std::false_type{});
        else
            launch_rows(std::true_type{});
    });
}
// Forward pass and pairs in one launch, if the rows and pairs are few: whether they were.
bool preference_few(int dtype, const forward_args& a, const preference_args& p, float* seq_logp, float* dlogp, float* loss, hipStream_t stream)
{
    const int64_t vecs = a.rows.vocab / per_of(dtype), each = vecs <= LANES_VECS ? 16 : vecs <= WAVE_VECS ? 4 : 1, workgroups = (a.rows.count + each - 1) / each;
    if (stream != nullptr || p.pairs > FEW_PAIRS || p.rows > FEW_PAIR_ROWS || workgroups < 1 || workgroups > DQ_ARRIVE_WORKGROUPS || vecs > 4096) return false;
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(workgroups)), dim3(THREADS), 0, stream, a, p, seq_logp, dlogp, loss); };
        if (each == 16)
            launch(k_preference_few<T, 16>);
        else if (each == 4)
            launch(k_preference_few<T, 64>);
        else
            launch(k_preference_few<T, 256>);
    });
    return true;
}
void backward(int dtype, const dq_rows& rows, const dq_rows& out, const int64_t* tokens, const float2* softmax, const float* dlogp, double temperature, double scale,
              hipStream_t stream)
{
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const auto launch = [&](auto kernel, int nv) {
            // a row has one vector less than its elements fill where it starts between two boundaries; its ends are the first slice's
            const uint32_t slices = static_cast<uint32_t>((rows.vocab / PER<T> + 64 * nv - 1) / (64 * nv));
            const uint32_t least = slices ? slices : 1;
            hipLaunchKernelGGL(kernel, grid_of((rows.count * least + 3) / 4), dim3(THREADS), 0, stream, rows, out, least, tokens, softmax, dlogp,
                               static_cast<float>(scale / temperature), exp2_scale(temperature));
        };
        const auto small = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid_of((rows.count + 15) / 16), dim3(THREADS), 0, stream, rows, out, tokens, softmax, dlogp, static_cast<float>(scale / temperature),
                               exp2_scale(temperature));
        };
        const int vecs = rows.vocab / PER<T>;
        if (vecs <= 16)
            small(k_small_gradient<T, 1>);
        else if (vecs <= 32)
            small(k_small_gradient<T, 2>);
        else if (vecs <= 64)
            small(k_small_gradient<T, 4>);
        else if (vecs <= 128)
            launch(k_token_gradient<T, 2>, 2);
        else
            launch(k_token_gradient<T, 4>, 4);
    });
}
constexpr int64_t FEW_ROWS = 512; // two for each CU: a row's own latency counts, so it gets more threads
// Workgroups of the fused kernel: a row each, or several small ones.
int64_t policy_workgroups(int dtype, int64_t rows, int64_t vecs)
{
    const int64_t each = vecs > WAVE_VECS ? 1 : vecs > LANES_VECS ? 4 : vecs > 64 && dtype == DQ_F32 ? 8 : 16;
    return (rows + each - 1) / each;
}
// How many sums are left to add, or 0 if the loss is written.
int64_t policy_gradient(int dtype, const dq_rows& rows, const dq_rows& out, const int64_t* tokens, const policy_args& p, double temperature, double scale, float* logp,
                        term_sums* sums, float* loss, void* slices, hipStream_t stream)
{
    const int64_t all_vecs = rows.vocab / per_of(dtype);
    const bool few = sliced(rows.count, all_vecs);
    const int64_t workgroups = few ? rows.count : policy_workgroups(dtype, rows.count, all_vecs);
    const bool arrive = stream == nullptr && workgroups <= MOST_ARRIVING;
    float* written = arrive ? loss : nullptr;
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const double inv_t = 1.0 / temperature;
        const float c = exp2_scale(temperature), factor = static_cast<float>(scale / temperature);
        const auto launch = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, grid_of(workgroups), dim3(threads), 0, stream, rows, out, tokens, p, inv_t, c, factor, logp, sums, written);
        };
        const int64_t vecs = rows.vocab / PER<T>;
        if (few) {
            const row_slices s = slices_of(rows.count, vecs, slices);
            const dim3 grid(static_cast<unsigned>(s.slices), static_cast<unsigned>(rows.count));
            const forward_args a = { rows, tokens, p.weights, inv_t, c, logp, nullptr, nullptr };
            hipLaunchKernelGGL(k_row_slices<T>, grid, dim3(THREADS), 0, stream, a, s, false);
            hipLaunchKernelGGL(k_policy_slices<T>, grid, dim3(THREADS), 0, stream, rows, out, tokens, p, inv_t, c, factor, logp, sums, written, s);
        } else if (vecs <= 16)
            launch(k_policy_fused<T, 16, 1, false>, 256);
        else if (vecs <= 32)
            launch(k_policy_fused<T, 16, 2, false>, 256);
        else if (vecs <= 64)
            launch(k_policy_fused<T, 16, 4, false>, 256);
        else if (vecs <= LANES_VECS && sizeof(T) == 2) // 16384 rows of 1000 bfloat16: 17.9 us; 32 lanes 18.6, a wavefront 23.2
            launch(k_policy_fused<T, 16, 8, false>, 256);
        else if (vecs <= LANES_VECS) // 65536 rows of 500 binary32: 54.7 us; 16 lanes 59.8
            launch(k_policy_fused<T, 32, 4, false>, 256);
        else if (vecs <= 256)
            launch(k_policy_fused<T, 64, 4, false>, 256);
        else if (vecs <= WAVE_VECS) // 16384 rows of 3000 and 4000 bfloat16: 41.4 and 52.5 us; two wavefronts 42.4 and 55.0
            launch(k_policy_fused<T, 64, 8, false>, 256);
        else if (vecs <= 1024)
            launch(k_policy_fused<T, 256, 4, false>, 256);
        else if (vecs <= 2048 && rows.count <= FEW_ROWS) // 100 rows of 12000 bfloat16: 8.3 us; 256 threads 9.3
            launch(k_policy_fused<T, 1024, 2, false>, 1024);
        else if (vecs <= 2048) // 8192 rows of 16384 bfloat16: 94 us; 512 threads 98, 1024 114
            launch(k_policy_fused<T, 256, 8, false>, 256);
        else if (vecs <= 4096 && sizeof(T) == 2 && rows.count > FEW_ROWS) // 2048 rows of 32768: 56 us; 256 threads 59, 1024 61
            launch(k_policy_fused<T, 512, 8, false>, 512);
        else if (vecs <= 4096) // 256 rows of 30000 bfloat16: 10.7 us, 512 threads 12.2; 8192 rows of 16384 binary32: 187, 256 and 512 threads 202
            launch(k_policy_fused<T, 1024, 4, false>, 1024);
        else if (vecs <= 8192)
            launch(k_policy_fused<T, 1024, 8, false>, 1024);
        else if (vecs <= 16384)
            launch(k_policy_fused<T, 1024, 16, false>, 1024);
        else
            launch(k_policy_fused<T, 1024, 16, true>, 1024);
    });
    return arrive ? 0 : workgroups;
}

// loss = scale * the sum of `count` term_sums, which lie in a workspace with room for SUM_SHARES more behind them
constexpr int64_t SUM_SHARES = 160;
static_assert(SUM_SHARES >= DQ_ARRIVE_WORKGROUPS, "a group's sum each");
constexpr int64_t SUM_AT_ONCE = 4096;
void sum_terms(term_sums* sums, int64_t count, double scale, float* loss, hipStream_t stream)
{
    if (count > SUM_AT_ONCE) {
        const int64_t each = (count + SUM_SHARES - 1) / SUM_SHARES;
        hipLaunchKernelGGL(k_sum_terms, dim3(SUM_SHARES), dim3(SUM_THREADS), 0, stream, sums, count, each, 1.0, sums + count, nullptr);
        sums += count;
        count = SUM_SHARES;
    }
    hipLaunchKernelGGL(k_sum_terms, dim3(1), dim3(SUM_THREADS), 0, stream, sums, count, count, scale, nullptr, loss);
}

} // namespace

extern "C" int64_t dq_token_logprob_workspace_bytes(int64_t rows, int64_t vocab)
{
    if (rows < 0 || rows > DQ_MAX_ROWS || vocab < 1 || vocab > INT32_MAX) return -1;
    return slices_room(rows, vocab) + 16;
}

extern "C" int dq_token_logprob(const dq_logits_t* logits, const int64_t* tokens_dev, double temperature, float* logp_dev, float* softmax_dev, void* workspace_dev,
                                void* hip_stream)
{
    dq_rows rows;
    const int rc = rows_of(logits, rows);
    if (rc != DQ_OK) return rc;
    if (!usable(temperature, 1.0)) return DQ_ERR_INVALID_ARG;
    if (rows.count == 0) return DQ_OK;
    if (!tokens_dev || !logp_dev || !workspace_dev || !aligned(tokens_dev, 8) || !aligned(logp_dev, 4) || !aligned(softmax_dev, 8) || !dq_aligned16(workspace_dev))
        return DQ_ERR_INVALID_ARG;
    dq_forget_earlier_errors();
    const forward_args a = { rows, tokens_dev, nullptr, 1.0 / temperature, exp2_scale(temperature), logp_dev, reinterpret_cast<float2*>(softmax_dev), nullptr };
    forward(logits->dtype, a, workspace_dev, static_cast<hipStream_t>(hip_stream));
    return launched();
}

extern "C" int dq_token_logprob_backward(const dq_logits_t* logits, const int64_t* tokens_dev, double temperature, const float* softmax_dev, const float* dlogp_dev,
                                         double grad_scale, const dq_logits_t* dlogits, void* hip_stream)
{
    dq_rows rows, out;
    int rc = rows_of(logits, rows);
    if (rc == DQ_OK) rc = gradient_of(dlogits, logits, out);
    if (rc != DQ_OK) return rc;
    if (!usable(temperature, grad_scale)) return DQ_ERR_INVALID_ARG;
    if (rows.count == 0) return DQ_OK;
    if (!tokens_dev || !softmax_dev || !dlogp_dev || !aligned(tokens_dev, 8) || !aligned(softmax_dev, 8) || !aligned(dlogp_dev, 4)) return DQ_ERR_INVALID_ARG;
    dq_forget_earlier_errors();
    backward(logits->dtype, rows, out, tokens_dev, reinterpret_cast<const float2*>(softmax_dev), dlogp_dev, temperature, grad_scale,
             static_cast<hipStream_t>(hip_stream));
    return launched();
}

extern "C" int64_t dq_policy_loss_workspace_bytes(int64_t rows, int64_t vocab)
{
    if (rows < 0 || rows > DQ_MAX_ROWS || vocab < 1 || vocab > INT32_MAX) return -1;
    return up((rows + SUM_SHARES) * static_cast<int64_t>(sizeof(term_sums))) + slices_room(rows, vocab);
}

extern "C" int dq_policy_loss(const dq_logits_t* logits, const int64_t* tokens_dev, double temperature, const float* old_logp_dev, const float* ref_logp_dev,
                              const float* advantages_dev, const float* weights_dev, double clip_low, double clip_high, double beta, double grad_scale,
                              float* loss_dev, float* logp_dev, const dq_logits_t* dlogits, void* workspace_dev, void* hip_stream)
{
    dq_rows rows, out;
    int rc = rows_of(logits, rows);
    if (rc == DQ_OK && dlogits) rc = gradient_of(dlogits, logits, out);
    if (rc != DQ_OK) return rc;
    if (!usable(temperature, grad_scale) || !(clip_low >= 0.0) || !(clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite(clip_high) || !(beta >= 0.0) ||
        !std::isfinite(beta))
        return DQ_ERR_INVALID_ARG;
    if (!loss_dev || !aligned(loss_dev, 4) || !workspace_dev || !dq_aligned16(workspace_dev) || (beta > 0.0 && !ref_logp_dev && rows.count)) return DQ_ERR_INVALID_ARG;
    if (rows.count) {
        if (!tokens_dev || !old_logp_dev || !advantages_dev || !weights_dev || !logp_dev || !aligned(tokens_dev, 8)) return DQ_ERR_INVALID_ARG;
        for (const void* p : { static_cast<const void*>(old_logp_dev), static_cast<const void*>(ref_logp_dev), static_cast<const void*>(advantages_dev),
                               static_cast<const void*>(weights_dev), static_cast<const void*>(logp_dev) })
            if (!aligned(p, 4)) return DQ_ERR_INVALID_ARG;
    }
    dq_forget_earlier_errors();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto* sums = static_cast<term_sums*>(workspace_dev);
    int64_t n_sums = 0;
    void* slices = static_cast<char*>(workspace_dev) + up((rows.count + SUM_SHARES) * static_cast<int64_t>(sizeof(term_sums)));
    const policy_args p = { old_logp_dev, ref_logp_dev, advantages_dev, weights_dev, static_cast<float>(1.0 - clip_low), static_cast<float>(1.0 + clip_high),
                            static_cast<float>(beta) };
    if (rows.count && dlogits) {
        n_sums = policy_gradient(logits->dtype, rows, out, tokens_dev, p, temperature, grad_scale, logp_dev, sums, loss_dev, slices, stream);
        if (n_sums == 0) return launched();
    } else if (rows.count) {
        const forward_args a = { rows, tokens_dev, weights_dev, 1.0 / temperature, exp2_scale(temperature), logp_dev, nullptr, nullptr };
        forward(logits->dtype, a, slices, stream);
        n_sums = (rows.count + THREADS - 1) / THREADS;
        hipLaunchKernelGGL(k_policy_rows, dim3(static_cast<unsigned>(n_sums)), dim3(THREADS), 0, stream, p, rows.count, static_cast<int64_t>(rows.vocab), tokens_dev, logp_dev, sums);
    }
    sum_terms(sums, n_sums, 1.0, loss_dev, stream);
    return launched();
}

extern "C" int64_t dq_preference_loss_workspace_bytes(int64_t rows, int64_t vocab, int64_t pairs)
{
    if (rows < 0 || rows > DQ_MAX_ROWS || vocab < 1 || vocab > INT32_MAX || pairs < 1 || pairs > DQ_MAX_ROWS) return -1;
    return up((pairs + SUM_SHARES) * static_cast<int64_t>(sizeof(term_sums))) + up(rows * 8) + 2 * up(rows * 4) + slices_room(rows, vocab) + 16;
}

extern "C" int dq_preference_loss(const dq_logits_t* logits, const int64_t* tokens_dev, double temperature, const int64_t* seq_start_dev, int64_t pairs,
                                  const float* ref_logp_dev, double beta, double label_smoothing, int average, double grad_scale, float* loss_dev,
                                  float* seq_logp_dev, const dq_logits_t* dlogits, void* workspace_dev, void* hip_stream)
{
    dq_rows rows, out;
    int rc = rows_of(logits, rows);
    if (rc == DQ_OK && dlogits) rc = gradient_of(dlogits, logits, out);
    if (rc != DQ_OK) return rc;
    if (!usable(temperature, grad_scale) || pairs < 1 || pairs > DQ_MAX_ROWS || !(beta >= 0.0) || !std::isfinite(beta) || !(label_smoothing >= 0.0) ||
        !(label_smoothing <= 1.0))
        return DQ_ERR_INVALID_ARG;
    if (!seq_start_dev || !loss_dev || !seq_logp_dev || !workspace_dev || !aligned(seq_start_dev, 8) || !aligned(ref_logp_dev, 4) || !aligned(loss_dev, 4) ||
        !aligned(seq_logp_dev, 4) || !dq_aligned16(workspace_dev))
        return DQ_ERR_INVALID_ARG;
    if (rows.count && (!tokens_dev || !aligned(tokens_dev, 8))) return DQ_ERR_INVALID_ARG;
    dq_forget_earlier_errors();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char* ws = static_cast<char*>(workspace_dev);
    auto* terms = reinterpret_cast<term_sums*>(ws);
    ws += up((pairs + SUM_SHARES) * static_cast<int64_t>(sizeof(term_sums)));
    auto* softmax = reinterpret_cast<float2*>(ws);
    ws += up(rows.count * 8);
    auto* logp = reinterpret_cast<float*>(ws);
    auto* dlogp = reinterpret_cast<float*>(ws + up(rows.count * 4));
    const preference_args p = { seq_start_dev, ref_logp_dev, pairs, rows.count, rows.vocab, static_cast<float>(beta), static_cast<float>(label_smoothing), average != 0 };
    const forward_args a = { rows, tokens_dev, nullptr, 1.0 / temperature, exp2_scale(temperature), logp, dlogits ? softmax : nullptr, dlogp };
    if (!preference_few(logits->dtype, a, p, seq_logp_dev, dlogp, loss_dev, stream)) {
        if (rows.count) forward(logits->dtype, a, reinterpret_cast<char*>(dlogp) + up(rows.count * 4), stream);
        const bool arrive = stream == nullptr && pairs <= MOST_ARRIVING;
        hipLaunchKernelGGL(k_preference_pairs, grid_of(pairs), dim3(THREADS), 0, stream, p, tokens_dev, logp, terms, seq_logp_dev, dlogp,
                           arrive ? loss_dev : nullptr);
        if (!arrive) sum_terms(terms, pairs, 1.0 / static_cast<double>(pairs), loss_dev, stream);
    }
    if (rows.count && dlogits) backward(logits->dtype, rows, out, tokens_dev, softmax, dlogp, temperature, grad_scale, stream);
    return launched();
}
