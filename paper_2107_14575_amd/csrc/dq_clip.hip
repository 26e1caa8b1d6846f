// The global norm over many tensors, and clipping to it: dq_grad_norm, dq_clip_grads, dq_clip_gather, dq_clip_norms.
//
// Two passes, since no element may be scaled before the last one has been squared.  The first sums squares in binary64 (those of binary32 values are
// exact there), one partial per workgroup; in the second every workgroup adds the partials in the same fixed order, so that all of them hold the
// same factor, and scales its share of the elements.  The memory binds both: 2^27 bfloat16 values in one tensor 128 us for 0.54 GB read and 0.27 written, of
// them 49 the first pass (5.4 TB/s) and 78 the second (6.9, a part of it from the last-level cache); in 290 tensors of all sizes 146.
#include "dq_internal.h"
#include "dq_vectors.h"

namespace {

constexpr int THREADS = 256;
constexpr int AT_ONCE = 4;                       // 16-byte vectors of a thread in flight
constexpr int PIECE = THREADS * AT_ONCE;         // vectors that a workgroup takes at a time: 16 KB
constexpr int MOST_WORKGROUPS = 2048;            // eight on each CU
constexpr int MOST_PARTIALS = MOST_WORKGROUPS;   // of one call
typedef uint32_t half_vec __attribute__((ext_vector_type(2)));
typedef half_vec half_vec_anywhere __attribute__((aligned(2)));
constexpr int TABLE = 160;                       // tensors of one launch: the table is an argument of the kernel

// Tensors as the kernels see them.  Tensor l is cut into pieces first[l] .. first[l + 1] - 1, each but the last of PIECE vectors' worth of elements.
struct clip_table {
    const void* src[TABLE];
    void* dst[TABLE];
    uint32_t first[TABLE];
    uint32_t last[TABLE]; // elements of the last piece << 2 | dtype
    uint32_t n, pieces;
};
static_assert(sizeof(clip_table) <= 4000, "beside the other arguments within 4 KB");

struct clip_piece {
    uint32_t tensor, index; // the index-th piece of the tensor
    int64_t len;            // of the tensor
    int dtype;
};
__device__ __forceinline__ clip_piece piece_of(const clip_table& t, uint32_t piece)
{
    uint32_t lo = 0, hi = t.n; // first[lo] <= piece < first[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        (t.first[mid] <= piece ? lo : hi) = mid;
    }
    const uint32_t end = lo + 1 < t.n ? t.first[lo + 1] : t.pieces;
    const int dtype = static_cast<int>(t.last[lo] & 3);
    const int64_t each = PIECE * (dtype == DQ_F32 ? 4 : 8);
    return { lo, piece - t.first[lo], static_cast<int64_t>(end - t.first[lo] - 1) * each + (t.last[lo] >> 2), dtype };
}

// the sum of a workgroup of N threads, in every one of them, in a fixed order
template <int N = THREADS>
__device__ __forceinline__ double workgroup_sum(double mine)
{
    __shared__ double parts[N / 64];
    for (int off = 32; off > 0; off /= 2) mine += __shfl_xor(mine, off, 64);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x / 64] = mine;
    __syncthreads();
    double sum = parts[0];
    for (int w = 1; w < N / 64; ++w) sum += parts[w];
    return sum;
}

// Binds a piece's tensor for one of THREADS threads: f(the typed source, its parts, this thread's first vector of the piece)
template <typename F>
__device__ __forceinline__ void with_piece(const clip_table& t, const clip_piece& p, int tid, F&& f)
{
    with_type(p.dtype, [&](auto type) {
        using T = decltype(type);
        const T* g = static_cast<const T*>(t.src[p.tensor]);
        const dq_parts<T, int64_t> parts(g, p.len);
        f(g, parts, static_cast<int64_t>(p.index) * PIECE + tid);
    });
}

// `mine` with the squares, in binary64, of one thread's share of the pieces from `piece` on, `step` apart.  Loads without the streaming hint: the second
// pass finds the last 256 MB in the last-level cache.
__device__ __forceinline__ void add_squares(double& mine, const clip_table& t, uint32_t piece, uint32_t step, int tid)
{
    for (; piece < t.pieces; piece += step) {
        const clip_piece p = piece_of(t, piece);
        with_piece(t, p, tid, [&](auto* g, const auto& parts, int64_t first) {
            using T = std::remove_cv_t<std::remove_pointer_t<decltype(g)>>;
            vec v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                for (int j = 0; j < 4; ++j) v[i][j] = 0;
                if (first + i * THREADS < parts.vecs) v[i] = load_vec<false>(g + parts.head + (first + i * THREADS) * PER<T>);
            }
            const int64_t end = p.index == 0 ? parts.end_of(tid, p.len) : -1;
            if (end >= 0) {
                const double d = static_cast<float>(g[end]);
                mine = fma(d, d, mine);
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                float x[PER<T>];
                unpack<T>(v[i], x);
                for (int j = 0; j < PER<T>; ++j) {
                    const double d = x[j];
                    mine = fma(d, d, mine);
                }
            }
        });
    }
}
// one partial sum for each workgroup
__global__ __launch_bounds__(THREADS) void k_squares(clip_table t, double* __restrict__ partials)
{
    double mine = 0.0;
    add_squares(mine, t, blockIdx.x, gridDim.x, threadIdx.x);
    const double sum = workgroup_sum(mine);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

__device__ __forceinline__ double clip_factor(double norm, double max_norm) { return norm <= max_norm ? 1.0 : max_norm / norm; }
// The factor as binary32 holds it, f = first * second: where it is below the normal numbers its products with a gradient that has grown so far are not, and
// `second` is the power of two that keeps `first` among them.  What that rounds in x * second is below the last place of the product.  Otherwise `second`
// is 1, whose product changes nothing.
struct clip_scale {
    float first, second;
    __device__ __forceinline__ explicit clip_scale(double f)
    {
        const double small = f < 0x1p-252 ? 0x1p-149 : f < 0x1p-126 ? 0x1p-126 : 1.0; // 1 for NaN
        first = static_cast<float>(f / small);
        second = static_cast<float>(small);
    }
    __device__ __forceinline__ float operator*(float x) const { return x * second * first; }
};

__device__ __forceinline__ double total_norm(const double* __restrict__ partials, int n)
{
    double mine = 0.0;
    for (int i = threadIdx.x; i < n; i += THREADS) mine += partials[i];
    return sqrt(workgroup_sum(mine));
}

__global__ __launch_bounds__(THREADS) void k_total(const double* __restrict__ partials, int n, float* __restrict__ norm)
{
    const double N = total_norm(partials, n);
    if (threadIdx.x == 0) *norm = static_cast<float>(N);
}

// One thread's share of the pieces times f, `back` pieces from the last one and `step` more each time: as the caches hold them.  ROW: into binary32, a tensor's
// first piece with the pads behind it.
template <bool ROW>
__device__ __forceinline__ void scale_pieces(const clip_table& t, const clip_scale& f, uint32_t back, uint32_t step, int tid)
{
    for (; back < t.pieces; back += step) {
        const clip_piece p = piece_of(t, t.pieces - 1 - back);
        with_piece(t, p, tid, [&](auto* g, const auto& parts, int64_t first) {
            using T = std::remove_cv_t<std::remove_pointer_t<decltype(g)>>;
            using Out = std::conditional_t<ROW, float, T>;
            Out* out = static_cast<Out*>(t.dst[p.tensor]);
            if (!ROW && f.first == 1.0f && f.second == 1.0f && static_cast<const void*>(out) == g) return;
            const int64_t end = p.index == 0 ? parts.end_of(tid, p.len) : -1;
            if (end >= 0) out[end] = static_cast<Out>(f * static_cast<float>(g[end]));
            if (ROW && p.index == 0 && p.len + tid < (p.len + DQ_GRANULE - 1) / DQ_GRANULE * DQ_GRANULE) out[p.len + tid] = static_cast<Out>(0.0f);
            g += parts.head;
            out += parts.head;
            if constexpr (ROW && sizeof(T) == 2) {
                // half a vector a lane, whose four binary32 values are one whole one: a store instruction then covers its lines (two stores of every
                // other 16 bytes: 2^27 values 268 -> 167 us)
                first = first * 2 - tid;
                half_vec v[2 * AT_ONCE];
#pragma unroll
                for (int i = 0; i < 2 * AT_ONCE; ++i)
                    if (first + i * THREADS < 2 * parts.vecs) v[i] = __builtin_nontemporal_load(reinterpret_cast<const half_vec_anywhere*>(g + (first + i * THREADS) * 4));
#pragma unroll
                for (int i = 0; i < 2 * AT_ONCE; ++i)
                    if (first + i * THREADS < 2 * parts.vecs) {
                        float x[8];
                        unpack<T>(vec{ v[i][0], v[i][1], 0, 0 }, x);
                        const float y[4] = { f * x[0], f * x[1], f * x[2], f * x[3] };
                        store_vec(out + (first + i * THREADS) * 4, pack<float>(y));
                    }
            } else {
                vec v[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (first + i * THREADS < parts.vecs) v[i] = load_vec<true>(g + (first + i * THREADS) * PER<T>);
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (first + i * THREADS < parts.vecs) {
                        float x[PER<T>];
                        unpack<T>(v[i], x);
                        for (int j = 0; j < PER<T>; ++j) x[j] = f * x[j];
                        store_vec(out + (first + i * THREADS) * PER<T>, pack<Out>(x));
                    }
            }
        });
    }
}

template <bool ROW>
__global__ __launch_bounds__(THREADS) void k_scale(clip_table t, const double* __restrict__ partials, int n_partials, double max_norm, float* __restrict__ norm)
{
    const double N = total_norm(partials, n_partials);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(N);
    scale_pieces<ROW>(t, clip_scale(clip_factor(N, max_norm)), blockIdx.x, gridDim.x, threadIdx.x);
}

// Both passes by one workgroup, its four quarters a piece each at a time: few pieces are two launches' latency.
constexpr uint32_t FEW_PIECES = 8;
constexpr int FEW_THREADS = 4 * THREADS;
template <bool ROW>
__global__ __launch_bounds__(FEW_THREADS) void k_clip_few(clip_table t, double max_norm, float* __restrict__ norm)
{
    const int quarter = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / THREADS)), tid = threadIdx.x % THREADS;
    double mine = 0.0;
    add_squares(mine, t, quarter, FEW_THREADS / THREADS, tid);
    const double N = sqrt(workgroup_sum<FEW_THREADS>(mine));
    if (threadIdx.x == 0) *norm = static_cast<float>(N);
    scale_pieces<ROW>(t, clip_scale(clip_factor(N, max_norm)), quarter, FEW_THREADS / THREADS, tid);
}

// A worker's norms in the registers of one workgroup, HELD of each of its threads.
constexpr int HELD_THREADS = 1024, HELD = 40;
__global__ __launch_bounds__(HELD_THREADS) void k_clip_norms(const float* __restrict__ norms, int n_seg, double max_norm, float* __restrict__ total, float* __restrict__ out)
{
    const int64_t row = static_cast<int64_t>(blockIdx.x) * n_seg;
    float v[HELD];
    double mine = 0.0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int l = i * HELD_THREADS + threadIdx.x;
        v[i] = l < n_seg ? norms[row + l] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) mine = fma(static_cast<double>(v[i]), static_cast<double>(v[i]), mine);
    const double N = sqrt(workgroup_sum<HELD_THREADS>(mine));
    if (threadIdx.x == 0) total[blockIdx.x] = static_cast<float>(N);
    const clip_scale f(clip_factor(N, max_norm));
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int l = i * HELD_THREADS + threadIdx.x;
        if (l < n_seg) out[row + l] = f * v[i];
    }
}

// More norms than that: a workgroup for each worker and share of its norms, which adds their squares ...
__global__ __launch_bounds__(THREADS) void k_norm_squares(const float* __restrict__ norms, int64_t n_seg, int shares, double* __restrict__ partials)
{
    const float* row = norms + static_cast<int64_t>(blockIdx.y) * n_seg;
    const dq_parts<float, int64_t> parts(row, n_seg);
    double mine = 0.0;
    const int64_t end = blockIdx.x == 0 ? parts.end_of(threadIdx.x, n_seg) : -1;
    if (end >= 0) mine = static_cast<double>(row[end]) * static_cast<double>(row[end]);
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * PIECE + threadIdx.x; at < parts.vecs; at += static_cast<int64_t>(shares) * PIECE) {
        vec v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            for (int j = 0; j < 4; ++j) v[i][j] = 0;
            if (at + i * THREADS < parts.vecs) v[i] = load_vec<false>(row + parts.head + (at + i * THREADS) * 4);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            for (int j = 0; j < 4; ++j) {
                const double d = __uint_as_float(v[i][j]);
                mine = fma(d, d, mine);
            }
    }
    const double sum = workgroup_sum(mine);
    if (threadIdx.x == 0) partials[blockIdx.y * shares + blockIdx.x] = sum;
}

// ... and scales them.
__global__ __launch_bounds__(THREADS) void k_norm_scale(const float* __restrict__ norms, int64_t n_seg, int shares, const double* __restrict__ partials,
                                                        double max_norm, float* __restrict__ total, float* __restrict__ out)
{
    const double N = total_norm(partials + blockIdx.y * shares, shares);
    if (blockIdx.x == 0 && threadIdx.x == 0) total[blockIdx.y] = static_cast<float>(N);
    const clip_scale f(clip_factor(N, max_norm));
    const float* row = norms + static_cast<int64_t>(blockIdx.y) * n_seg;
    float* to = out + static_cast<int64_t>(blockIdx.y) * n_seg;
    const dq_parts<float, int64_t> parts(row, n_seg);
    const int64_t end = blockIdx.x == 0 ? parts.end_of(threadIdx.x, n_seg) : -1;
    if (end >= 0) to[end] = f * row[end];
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * PIECE + threadIdx.x; at < parts.vecs; at += static_cast<int64_t>(shares) * PIECE) {
        vec v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (at + i * THREADS < parts.vecs) v[i] = load_vec<true>(row + parts.head + (at + i * THREADS) * 4);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (at + i * THREADS < parts.vecs) {
                const float x[4] = { f * __uint_as_float(v[i][0]), f * __uint_as_float(v[i][1]), f * __uint_as_float(v[i][2]), f * __uint_as_float(v[i][3]) };
                store_vec(to + parts.head + (at + i * THREADS) * 4, pack<float>(x));
            }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------
constexpr int64_t MAX_LEN = INT64_C(1) << 40;
constexpr int32_t MAX_TENSORS = 1 << 18;
static_assert(MAX_TENSORS <= TABLE * MOST_PARTIALS, "a workgroup for each table");

// A call's tensors, table after table, in their order; tensors without elements are in none.
struct tensors {
    const void* const* src;
    void* const* dst;     // null: no destination, or the row
    float* row;
    const dq_plan* plan;  // of the row
    const int64_t* len;
    const int32_t* dtype;
    int32_t n;

    int64_t each_of(int32_t l) const { return PIECE * (dtype[l] == DQ_F32 ? 4 : 8); }
    int64_t pieces_of(int32_t l) const { return (len[l] + each_of(l) - 1) / each_of(l); }
    int check() const
    {
        if (n < 0 || n > MAX_TENSORS || (n && (!src || !len || !dtype))) return DQ_ERR_INVALID_ARG;
        int64_t pieces = 0;
        for (int32_t l = 0; l < n; ++l) {
            if (len[l] < 0 || len[l] > MAX_LEN || dtype[l] < DQ_F32 || dtype[l] > DQ_BF16) return DQ_ERR_INVALID_ARG;
            const size_t size = dtype[l] == DQ_F32 ? 4 : 2;
            if (len[l] && (!src[l] || !aligned(src[l], size) || (dst && (!dst[l] || !aligned(dst[l], size))))) return DQ_ERR_INVALID_ARG;
            pieces += pieces_of(l);
            if (pieces > INT32_MAX) return DQ_ERR_INVALID_ARG;
        }
        return DQ_OK;
    }
    // the next table from tensor `from` on; the tensor after its last one
    int32_t fill(clip_table& t, int32_t from) const
    {
        t.n = t.pieces = 0;
        int32_t l = from;
        for (; l < n && t.n < TABLE; ++l) {
            if (!len[l]) continue;
            t.src[t.n] = src[l];
            t.dst[t.n] = dst ? dst[l] : row ? row + plan->seg_start[l] : nullptr;
            const int64_t pieces = pieces_of(l);
            t.last[t.n] = static_cast<uint32_t>(len[l] - (pieces - 1) * each_of(l)) << 2 | static_cast<uint32_t>(dtype[l]);
            t.first[t.n++] = t.pieces;
            t.pieces += static_cast<uint32_t>(pieces);
        }
        return l;
    }
    int tables() const
    {
        int with = 0;
        for (int32_t l = 0; l < n; ++l) with += len[l] != 0;
        return (with + TABLE - 1) / TABLE;
    }
};

// Partial sums of squares of all tables; their number.  Each launch gets an equal part of MOST_PARTIALS, down to one.  More of them gain nothing where tables are many: 700 and 1300
// tensors of 2^27 bfloat16 values in all take 162 and 293 us, with eight times the partials 160 and 294, since the host's work for their arguments binds.
int squares(const tensors& all, double* partials, hipStream_t stream)
{
    const int tables = all.tables();
    const uint32_t most = tables ? MOST_PARTIALS / tables : 0;
    int used = 0;
    clip_table t;
    for (int32_t l = 0; l < all.n;) {
        l = all.fill(t, l);
        if (!t.n) break;
        const uint32_t grid = t.pieces < most ? t.pieces : most;
        hipLaunchKernelGGL(k_squares, dim3(grid), dim3(THREADS), 0, stream, t, partials + used);
        used += static_cast<int>(grid);
    }
    return used;
}

template <bool ROW>
int clip(const tensors& all, double max_norm, float* norm, void* workspace, hipStream_t stream)
{
    clip_table t;
    if (all.tables() == 1) {
        all.fill(t, 0);
        if (t.pieces <= FEW_PIECES) { // 1000 values in each of three tensors 9.0 -> 5.9 us
            hipLaunchKernelGGL(k_clip_few<ROW>, dim3(1), dim3(FEW_THREADS), 0, stream, t, max_norm, norm);
            return launched();
        }
    }
    auto* partials = static_cast<double*>(workspace);
    const int used = squares(all, partials, stream);
    bool first = true;
    for (int32_t l = 0; l < all.n;) {
        l = all.fill(t, l);
        if (!t.n) break;
        const uint32_t grid = t.pieces < MOST_WORKGROUPS ? t.pieces : MOST_WORKGROUPS;
        hipLaunchKernelGGL(k_scale<ROW>, dim3(grid), dim3(THREADS), 0, stream, t, partials, used, max_norm, first ? norm : nullptr);
        first = false;
    }
    if (first) hipLaunchKernelGGL(k_total, dim3(1), dim3(THREADS), 0, stream, partials, 0, norm);
    return launched();
}

bool usable(double max_norm) { return max_norm >= 0.0; } // infinity: no bound

} // namespace

extern "C" int64_t dq_clip_workspace_bytes(void) { return MOST_PARTIALS * 8; }

extern "C" int dq_grad_norm(const void* const* grads_host, const int64_t* len_host, const int32_t* dtype_host, int32_t n, float* norm_dev, void* workspace_dev,
                            void* hip_stream)
{
    const tensors all = { grads_host, nullptr, nullptr, nullptr, len_host, dtype_host, n };
    const int rc = all.check();
    if (rc != DQ_OK) return rc;
    if (!norm_dev || !workspace_dev || !aligned(norm_dev, 4) || !dq_aligned16(workspace_dev)) return DQ_ERR_INVALID_ARG;
    dq_forget_earlier_errors();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto* partials = static_cast<double*>(workspace_dev);
    const int used = squares(all, partials, stream);
    hipLaunchKernelGGL(k_total, dim3(1), dim3(THREADS), 0, stream, partials, used, norm_dev);
    return launched();
}

extern "C" int dq_clip_grads(const void* const* grads_host, void* const* out_host, const int64_t* len_host, const int32_t* dtype_host, int32_t n, double max_norm,
                             float* norm_dev, void* workspace_dev, void* hip_stream)
{
    if (n > 0 && !out_host) return DQ_ERR_INVALID_ARG;
    const tensors all = { grads_host, out_host, nullptr, nullptr, len_host, dtype_host, n };
    const int rc = all.check();
    if (rc != DQ_OK) return rc;
    if (!usable(max_norm) || !norm_dev || !workspace_dev || !aligned(norm_dev, 4) || !dq_aligned16(workspace_dev))
        return DQ_ERR_INVALID_ARG;
    dq_forget_earlier_errors();
    return clip<false>(all, max_norm, norm_dev, workspace_dev, static_cast<hipStream_t>(hip_stream));
}

extern "C" int dq_clip_gather(const dq_plan_t* plan, const void* const* grads_host, const int32_t* dtype_host, double max_norm, float* norm_dev, float* row_dev,
                              void* workspace_dev, void* hip_stream)
{
    if (!plan || !row_dev || !dq_aligned16(row_dev)) return DQ_ERR_INVALID_ARG;
    const tensors all = { grads_host, nullptr, row_dev, plan, plan->seg_len, dtype_host, plan->n_seg };
    int rc = all.check();
    if (rc != DQ_OK) return rc;
    if (!usable(max_norm) || !norm_dev || !workspace_dev || !aligned(norm_dev, 4) || !dq_aligned16(workspace_dev))
        return DQ_ERR_INVALID_ARG;
    rc = dq_plan_check_device(plan);
    if (rc != DQ_OK) return rc;
    return clip<true>(all, max_norm, norm_dev, workspace_dev, static_cast<hipStream_t>(hip_stream));
}

namespace {
// workgroups for each worker's norms: 16 KB each, eight on each CU for all the workers together
int shares_of(int M, int64_t n_seg)
{
    const int64_t by_size = (n_seg + 4 * PIECE - 1) / (4 * PIECE), most = MOST_WORKGROUPS / M;
    return static_cast<int>(by_size < 1 ? 1 : by_size < most ? by_size : most);
}
} // namespace

extern "C" int64_t dq_clip_norms_workspace_bytes(int M, int64_t n_seg)
{
    if (M < 1 || M > DQ_MAX_WORKERS || n_seg < 0 || n_seg > MAX_LEN) return -1;
    return static_cast<int64_t>(M) * shares_of(M, n_seg) * 8;
}

extern "C" int dq_clip_norms(const float* norms_dev, int M, int64_t n_seg, double max_norm, float* total_dev, float* out_dev, void* workspace_dev, void* hip_stream)
{
    if (M < 1 || M > DQ_MAX_WORKERS || n_seg < 0 || n_seg > MAX_LEN || !usable(max_norm) || !total_dev || !aligned(total_dev, 4)) return DQ_ERR_INVALID_ARG;
    if (n_seg && (!norms_dev || !out_dev || !aligned(norms_dev, 4) || !aligned(out_dev, 4))) return DQ_ERR_INVALID_ARG;
    if (!workspace_dev || !dq_aligned16(workspace_dev)) return DQ_ERR_INVALID_ARG;
    dq_forget_earlier_errors();
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (n_seg <= HELD * HELD_THREADS) { // one launch for two: 16 x 32771 norms 8.8 -> 5.4 us
        hipLaunchKernelGGL(k_clip_norms, dim3(static_cast<unsigned>(M)), dim3(HELD_THREADS), 0, stream, norms_dev, static_cast<int>(n_seg), max_norm, total_dev, out_dev);
        return launched();
    }
    const int shares = shares_of(M, n_seg);
    const dim3 grid(static_cast<unsigned>(shares), static_cast<unsigned>(M));
    auto* partials = static_cast<double*>(workspace_dev);
    hipLaunchKernelGGL(k_norm_squares, grid, dim3(THREADS), 0, stream, norms_dev, n_seg, shares, partials);
    hipLaunchKernelGGL(k_norm_scale, grid, dim3(THREADS), 0, stream, norms_dev, n_seg, shares, partials, max_norm, total_dev, out_dev);
    return launched();
}
