// The norm over all elements of many tensors, and clipping to it.
//
//   norm = sqrt(sum g^2) or max |g|;   factor = norm <= max_norm ? 1 : max_norm / norm;   to = factor * from
//
// Tensors are cut into tiles of TILE_VECS 16-byte accesses; a launch's workgroups take tiles in turn, add the squares in fp64 (the square
// of an fp32 number is exact there and cannot overflow) and store one partial result each, which are added in a fixed order: no atomics,
// bitwise reproducible.  The workgroups of the scaling pass each form that last sum by themselves, which saves a launch between the two
// passes.  The list of tensors travels in the kernel arguments (4 KB hold LIST tensors; a longer list takes several launches), so
// that nothing has to be copied to the device and a call can be captured.  Bound by bytes: 577 M bf16 elements in 288 tensors 605 us, the norm at
// 5.2 to 5.9 TB/s and the scaling pass at 5.9; 144 M fp32 elements 280 us, where the second pass finds part of what the first read in the cache.
#include "common.h"
#include "values.h"

#include <cmath>

namespace slicegcn {

namespace {

constexpr int THREADS = 256;
constexpr int TILE_VECS = 4 * THREADS; // 16-byte accesses per tile
constexpr int LIST = 144;              // tensors per launch
// Workgroups of a launch: one per tile while those fit the chip at once, else two per CU that take tiles in turn.  Clipping 13 M bf16 elements (1582
// tiles) 18.5 us, with 512 workgroups 23.7; 144 M fp32 elements in one launch 283 us with 512, 293 with 1024, 317 with 2048.
inline int32_t blocks_for(int64_t tiles) { return (int32_t)(tiles <= 2048 ? tiles : 512); }

struct TensorRange { // the tensors of one launch; a tensor's tiles are [first[i], first[i + 1])
    const void *from[LIST];
    void *to[LIST];
    uint64_t count[LIST]; // elements, type in the upper bits
    uint32_t first[LIST + 1];
};
constexpr int TYPE_SHIFT = 56;

struct LaunchPart {
    int32_t tensors;
    uint32_t tiles;
};

__device__ inline double wave_sum(double v)
{
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s, 64);
    return v;
}

__device__ inline uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, s, 64));
    return v;
}

// The running result of a thread: a sum of squares, or the largest |g| as bits (which order like the numbers, NaN above all of them)
template <int KIND> struct Running;
template <> struct Running<SLICEGCN_NORM_TWO> {
    double v = 0.0;
    __device__ void add(float g) { v = fma((double)g, (double)g, v); }
    __device__ void join(uint64_t o) { v += __longlong_as_double((long long)o); }
    __device__ uint64_t bits() const { return (uint64_t)__double_as_longlong(v); }
    __device__ void over_wave() { v = wave_sum(v); }
    __device__ double norm() const { return sqrt(v); }
};
template <> struct Running<SLICEGCN_NORM_MAX> {
    uint32_t v = 0;
    __device__ void add(float g) { v = max(v, __float_as_uint(g) & 0x7fffffffu); }
    __device__ void join(uint64_t o) { v = max(v, (uint32_t)o); }
    __device__ uint64_t bits() const { return v; }
    __device__ void over_wave() { v = wave_max(v); }
    __device__ double norm() const { return (double)__uint_as_float(v); }
};

// Over the workgroup's WAVES wavefronts, in every thread
template <int WAVES, int KIND> __device__ inline void over_block(Running<KIND> &r, uint64_t *shared)
{
    r.over_wave();
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = r.bits();
    __syncthreads();
    Running<KIND> all;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all.join(shared[w]);
    r = all;
}

// f(element type, tensor, its first vector) for the tiles first, first + step, ... below `tiles`, the last one first where BACK
template <bool BACK, class F> __device__ inline void for_tiles(const TensorRange &list, int tensors, uint32_t first, uint32_t step, uint32_t tiles, F f)
{
    if (first >= tiles) return;
    const uint32_t count = (tiles - first + step - 1) / step, from = BACK ? first + (count - 1) * step : first;
    int t = 0, hi = tensors; // the tensor that holds the tile: the last one that starts at or before it
    while (hi - t > 1) {
        const int mid = (t + hi) / 2;
        if (list.first[mid] <= from) t = mid;
        else hi = mid;
    }
    for (uint32_t k = 0; k < count; ++k) {
        const uint32_t tile = BACK ? from - k * step : from + k * step;
        if (BACK)
            while (list.first[t] > tile) --t;
        else
            while (list.first[t + 1] <= tile) ++t; // also past tensors without tiles
        const int64_t v0 = (int64_t)(tile - list.first[t]) * TILE_VECS;
        const int type = (int)(list.count[t] >> TYPE_SHIFT);
        if (type == SLICEGCN_F32) f(float(), t, v0);
        else if (type == SLICEGCN_BF16) f(bf16(), t, v0);
        else f(f16(), t, v0);
    }
}

__device__ inline int64_t elements(const TensorRange &list, int t) { return (int64_t)(list.count[t] & (((uint64_t)1 << TYPE_SHIFT) - 1)); }

// The accesses of a tile by `threads` threads, of which this is the thread-th: whole(vector index, value) and rest(element index) for the last few
template <class T, int THREADS_, class W, class R>
__device__ inline void tile_accesses(const T *p, int64_t count, int64_t v0, int thread, W whole, R rest)
{
    constexpr int V = 16 / sizeof(T), N = TILE_VECS / THREADS_;
    const int64_t vecs = count / V;
    if (v0 + TILE_VECS <= vecs) {
        typename VecOf<T, V>::type x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = load_vec<T, V>(p + (v0 + thread + i * THREADS_) * V);
#pragma unroll
        for (int i = 0; i < N; ++i) whole(v0 + thread + i * THREADS_, x[i]);
        return;
    }
    for (int64_t v = v0 + thread; v < vecs; v += THREADS_) whole(v, load_vec<T, V>(p + v * V));
    for (int64_t i = vecs * V + thread; i < count; i += THREADS_) rest(i);
}

template <class T, int THREADS_, int KIND>
__device__ inline void add_tile(const TensorRange &list, int t, int64_t v0, int thread, Running<KIND> &r)
{
    const T *p = static_cast<const T *>(list.from[t]);
    tile_accesses<T, THREADS_>(p, elements(list, t), v0, thread,
                               [&](int64_t, const auto &x) {
#pragma unroll
                                   for (int j = 0; j < 16 / (int)sizeof(T); ++j) r.add((float)x[j]);
                               },
                               [&](int64_t i) { r.add((float)p[i]); });
}

template <bool PAST, class T, int THREADS_>
__device__ inline void scale_tile(const TensorRange &list, int t, int64_t v0, int thread, float f)
{
    constexpr int V = 16 / sizeof(T);
    const T *p = static_cast<const T *>(list.from[t]); // from and to may be the same tensor: a thread reads what it writes
    T *q = static_cast<T *>(list.to[t]);
    if (p == q && f == 1.f) return;
    tile_accesses<T, THREADS_>(p, elements(list, t), v0, thread,
                               [&](int64_t v, const auto &x) {
                                   float o[V];
#pragma unroll
                                   for (int j = 0; j < V; ++j) o[j] = f * (float)x[j];
                                   store_result<PAST, T, V>(q + v * V, o);
                               },
                               [&](int64_t i) { q[i] = (T)(f * (float)p[i]); });
}

template <int KIND>
__global__ __launch_bounds__(THREADS) void norm_partial_kernel(const TensorRange list, const LaunchPart part, uint64_t *__restrict__ partial)
{
    __shared__ uint64_t shared[THREADS / 64];
    Running<KIND> r;
    for_tiles<false>(list, part.tensors, blockIdx.x, gridDim.x, part.tiles,
                     [&](auto zero, int t, int64_t v0) { add_tile<decltype(zero), THREADS>(list, t, v0, threadIdx.x, r); });
    over_block<THREADS / 64>(r, shared);
    if (threadIdx.x == 0) partial[blockIdx.x] = r.bits();
}

template <int KIND> __device__ inline Running<KIND> join_partials(const uint64_t *__restrict__ partial, int32_t partials, uint64_t *shared)
{
    Running<KIND> r;
    for (int32_t i = threadIdx.x; i < partials; i += THREADS) r.join(partial[i]);
    over_block<THREADS / 64>(r, shared);
    return r;
}

template <int KIND>
__device__ inline float store_norm(const Running<KIND> &r, double max_norm, bool store, float *__restrict__ norm, float *__restrict__ factor)
{
    const double n = r.norm();
    const float f = n <= max_norm ? 1.f : (float)(max_norm / n);
    if (store) {
        if (norm) *norm = (float)n;
        if (factor) *factor = f;
    }
    return f;
}

template <int KIND>
__global__ __launch_bounds__(THREADS) void norm_final_kernel(const uint64_t *__restrict__ partial, int32_t partials, double max_norm,
                                                             float *__restrict__ norm, float *__restrict__ factor)
{
    __shared__ uint64_t shared[THREADS / 64];
    const Running<KIND> r = join_partials<KIND>(partial, partials, shared);
    store_norm<KIND>(r, max_norm, threadIdx.x == 0, norm, factor);
}

// The tiles in the opposite order of the pass before: what that read last may still lie in the last-level cache (256 MB).
template <int KIND, bool PAST>
__global__ __launch_bounds__(THREADS) void clip_kernel(const TensorRange list, const LaunchPart part, const uint64_t *__restrict__ partial,
                                                       int32_t partials, double max_norm, float *__restrict__ norm, float *__restrict__ factor)
{
    __shared__ uint64_t shared[THREADS / 64];
    const Running<KIND> r = join_partials<KIND>(partial, partials, shared);
    const float f = store_norm<KIND>(r, max_norm, blockIdx.x == 0 && threadIdx.x == 0, norm, factor);
    for_tiles<true>(list, part.tensors, blockIdx.x, gridDim.x, part.tiles,
                    [&](auto zero, int t, int64_t v0) { scale_tile<PAST, decltype(zero), THREADS>(list, t, v0, threadIdx.x, f); });
}

// Few tiles: one workgroup, a wavefront per tile, does all of it in one launch.
constexpr int SMALL_THREADS = 1024, SMALL_TILES = 2 * SMALL_THREADS / 64;
template <int KIND>
__global__ __launch_bounds__(SMALL_THREADS) void clip_small_kernel(const TensorRange list, int tensors, uint32_t tiles, double max_norm,
                                                                   float *__restrict__ norm, float *__restrict__ factor, bool scale)
{
    __shared__ uint64_t shared[SMALL_THREADS / 64];
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Running<KIND> r;
    for_tiles<false>(list, tensors, wave, SMALL_THREADS / 64, tiles,
                     [&](auto zero, int t, int64_t v0) { add_tile<decltype(zero), 64>(list, t, v0, lane, r); });
    over_block<SMALL_THREADS / 64>(r, shared);
    const float f = store_norm<KIND>(r, max_norm, threadIdx.x == 0, norm, factor);
    if (!scale) return;
    for_tiles<false>(list, tensors, wave, SMALL_THREADS / 64, tiles,
                     [&](auto zero, int t, int64_t v0) { scale_tile<false, decltype(zero), 64>(list, t, v0, lane, f); });
}

int64_t tiles_of(const slicegcn_tensor &t)
{
    const int64_t per_tile = TILE_VECS * 16 / type_bytes(t.type);
    return (t.count + per_tile - 1) / per_tile;
}

struct CallPlan {
    int64_t tiles = 0;
    int32_t partials = 0; // workgroups over all launches
    bool small = false;   // one launch does everything
};

int check_tensors(const char *what, const slicegcn_tensor *t, int32_t count)
{
    SG_REQUIRE(count >= 0 && (t || count == 0), SLICEGCN_EINVAL, "%s: no list of tensors", what);
    for (int32_t i = 0; i < count; ++i) {
        SG_REQUIRE(known_type(t[i].type), SLICEGCN_EINVAL, "%s: tensor %d has unknown type %d", what, i, t[i].type);
        SG_REQUIRE(t[i].count >= 0 && t[i].count < ((int64_t)1 << 48), SLICEGCN_EINVAL, "%s: tensor %d has a bad number of elements", what, i);
        SG_REQUIRE((t[i].data || t[i].count == 0) && aligned_for(t[i].data, t[i].type), SLICEGCN_EINVAL,
                   "%s: tensor %d is NULL or misaligned", what, i);
    }
    return SLICEGCN_OK;
}

// Calls f(first tensor, tensors, tiles) for the tensors of each launch, the last launch first where `back`
template <class F> int for_launches(const slicegcn_tensor *t, int32_t count, bool back, F f)
{
    const int32_t launches = (count + LIST - 1) / LIST;
    for (int32_t k = 0; k < launches; ++k) {
        const int32_t first = (back ? launches - 1 - k : k) * LIST, n = count - first < LIST ? count - first : LIST;
        int64_t tiles = 0;
        for (int32_t i = 0; i < n; ++i) tiles += tiles_of(t[first + i]);
        SG_REQUIRE(tiles <= UINT32_MAX, SLICEGCN_ERANGE, "global_norm: more than 2^32 tiles of 16 KB");
        if (tiles > 0)
            if (int rc = f(first, n, tiles)) return rc;
    }
    return SLICEGCN_OK;
}

int plan_call(const slicegcn_tensor *t, int32_t count, CallPlan *plan)
{
    for (int32_t i = 0; i < count; ++i) plan->tiles += tiles_of(t[i]);
    plan->small = plan->tiles <= SMALL_TILES && count <= LIST;
    if (plan->small) return SLICEGCN_OK;
    return for_launches(t, count, false, [&](int32_t, int32_t, int64_t tiles) {
        plan->partials += blocks_for(tiles);
        return SLICEGCN_OK;
    });
}

// Tensors [first, first + n) as a kernel argument
TensorRange make_list(const slicegcn_tensor *from, const slicegcn_tensor *to, int32_t first, int32_t n)
{
    TensorRange list;
    uint32_t at = 0;
    for (int32_t i = 0; i < n; ++i) {
        list.from[i] = from[first + i].data;
        list.to[i] = to ? to[first + i].data : from[first + i].data;
        list.count[i] = (uint64_t)from[first + i].count | ((uint64_t)from[first + i].type << TYPE_SHIFT);
        list.first[i] = at;
        at += (uint32_t)tiles_of(from[first + i]);
    }
    for (int32_t i = n; i < LIST; ++i) list.from[i] = nullptr, list.to[i] = nullptr, list.count[i] = 0;
    for (int32_t i = n; i <= LIST; ++i) list.first[i] = at;
    return list;
}

// Launches a kernel over all tensors: launch(list, part, blocks, blocks launched before)
template <class F> int launch_lists(const slicegcn_tensor *from, const slicegcn_tensor *to, int32_t count, bool back, F launch)
{
    int32_t before = 0;
    return for_launches(from, count, back, [&](int32_t first, int32_t n, int64_t tiles) {
        const LaunchPart part{n, (uint32_t)tiles};
        const int32_t blocks = blocks_for(tiles);
        launch(make_list(from, to, first, n), part, blocks, before);
        SG_LAUNCH_CHECK();
        before += blocks;
        return SLICEGCN_OK;
    });
}

int check_call(const char *what, const slicegcn_tensor *t, int32_t count, int32_t kind, double max_norm, CallPlan *plan, void *ws, size_t ws_bytes)
{
    if (int rc = check_tensors(what, t, count)) return rc;
    SG_REQUIRE(kind == SLICEGCN_NORM_TWO || kind == SLICEGCN_NORM_MAX, SLICEGCN_EINVAL, "%s: unknown kind %d", what, kind);
    SG_REQUIRE(max_norm >= 0.0, SLICEGCN_EINVAL, "%s: max_norm is negative or no number", what);
    if (int rc = plan_call(t, count, plan)) return rc;
    const size_t need = slicegcn_global_norm_workspace_bytes(t, count);
    SG_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SLICEGCN_EINVAL, "%s: misaligned workspace", what);
    SG_REQUIRE(need == 0 || (ws && ws_bytes >= need), SLICEGCN_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need);
    return SLICEGCN_OK;
}

template <int KIND>
int call(const slicegcn_tensor *from, const slicegcn_tensor *to, int32_t count, bool scale, const CallPlan &plan, double max_norm, float *norm,
         float *factor, uint64_t *ws, hipStream_t stream)
{
    if (plan.small) {
        clip_small_kernel<KIND><<<1, SMALL_THREADS, 0, stream>>>(make_list(from, to, 0, count), count, (uint32_t)plan.tiles, max_norm, norm, factor, scale);
        SG_LAUNCH_CHECK();
        return SLICEGCN_OK;
    }
    if (int rc = launch_lists(from, nullptr, count, false, [&](const TensorRange &list, const LaunchPart &part, int32_t blocks, int32_t before) {
            norm_partial_kernel<KIND><<<blocks, THREADS, 0, stream>>>(list, part, ws + before);
        }))
        return rc;
    if (!scale || plan.tiles == 0) {
        norm_final_kernel<KIND><<<1, THREADS, 0, stream>>>(ws, plan.partials, max_norm, norm, factor);
        SG_LAUNCH_CHECK();
        return SLICEGCN_OK;
    }
    return launch_lists(from, to, count, true, [&](const TensorRange &list, const LaunchPart &part, int32_t blocks, int32_t before) {
        with_flag(past_cache(plan.tiles, TILE_VECS * 4, SLICEGCN_F32), [&](auto past) {
            clip_kernel<KIND, decltype(past)::value><<<blocks, THREADS, 0, stream>>>(list, part, ws, plan.partials, max_norm, before ? nullptr : norm,
                                                                                    before ? nullptr : factor);
        });
    });
}

} // namespace
} // namespace slicegcn

using namespace slicegcn;

extern "C" size_t slicegcn_global_norm_workspace_bytes(const slicegcn_tensor *tensors, int32_t count)
{
    CallPlan plan;
    if (check_tensors("global_norm_workspace_bytes", tensors, count) || plan_call(tensors, count, &plan)) return 0;
    return (size_t)round_up(8 * (int64_t)plan.partials, 256);
}

extern "C" int slicegcn_global_norm(const slicegcn_tensor *tensors, int32_t count, int32_t kind, double max_norm, float *norm, float *factor,
                                    void *ws, size_t ws_bytes, void *stream)
{
    CallPlan plan;
    SG_REQUIRE(norm != nullptr, SLICEGCN_EINVAL, "global_norm: NULL norm");
    if (int rc = check_call("global_norm", tensors, count, kind, factor ? max_norm : 0.0, &plan, ws, ws_bytes)) return rc;
    ProfScope prof(SLICEGCN_PROF_CLIP, count, as_stream(stream));
    auto *w = static_cast<uint64_t *>(ws);
    return kind == SLICEGCN_NORM_TWO ? call<SLICEGCN_NORM_TWO>(tensors, nullptr, count, false, plan, max_norm, norm, factor, w, as_stream(stream))
                                     : call<SLICEGCN_NORM_MAX>(tensors, nullptr, count, false, plan, max_norm, norm, factor, w, as_stream(stream));
}

extern "C" int slicegcn_clip(const slicegcn_tensor *from, const slicegcn_tensor *to, int32_t count, int32_t kind, double max_norm, float *norm,
                             float *factor, void *ws, size_t ws_bytes, void *stream)
{
    CallPlan plan;
    if (int rc = check_call("clip", from, count, kind, max_norm, &plan, ws, ws_bytes)) return rc;
    if (to) {
        if (int rc = check_tensors("clip", to, count)) return rc;
        for (int32_t i = 0; i < count; ++i)
            SG_REQUIRE(to[i].count == from[i].count && to[i].type == from[i].type, SLICEGCN_EINVAL,
                       "clip: tensor %d differs in elements or type from what it is clipped from", i);
    }
    ProfScope prof(SLICEGCN_PROF_CLIP, count, as_stream(stream));
    auto *w = static_cast<uint64_t *>(ws);
    return kind == SLICEGCN_NORM_TWO ? call<SLICEGCN_NORM_TWO>(from, to, count, true, plan, max_norm, norm, factor, w, as_stream(stream))
                                     : call<SLICEGCN_NORM_MAX>(from, to, count, true, plan, max_norm, norm, factor, w, as_stream(stream));
}
