// One AdamW step over many tensors, states in 32 bits or in 8 with a power of two per block.
//
//   g = factor grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  p -= lr decay p + lr (m / c1) / (sqrt(v / c2) + eps)
//
// A thread takes 8 consecutive elements, so that 16 lanes hold a block of 128 and find its largest values among themselves.  Tensors are cut into tiles of one
// pass of a workgroup, which workgroups take in turn; the list of tensors travels in the kernel arguments (4 KB hold LIST tensors; a longer list takes
// several launches), so that nothing has to be copied to the device and a call can be captured.
//
// Bound by bytes: 768 M parameters in bf16 with fp32 masters, states in 8 bits: 1.86 ms, 4.95 TB/s.
//
// States in 8 bits: a mean that moves by 1 - b2 = 0.001 of its distance a step cannot be kept with a step size of 1/8 by rounding to nearest: it would not move at all.
// Values are therefore rounded up or down by chance, which keeps the mean; and scales are powers of two, so that the grid of a block stays where it is while the
// exponent of its largest value does, and a value that lies on the grid gains noise from its own change alone (a scale that followed the largest
// value itself would move the grid, and all of the block's values be rounded anew, every step).
#include "common.h"
#include "values.h"

#include <cfloat>
#include <cmath>

namespace slicegcn {

namespace {

constexpr int THREADS = 256, EACH = 8, TILE = THREADS * EACH, BLOCK = SLICEGCN_STATE_BLOCK;
constexpr int LANES = BLOCK / EACH; // lanes that hold a block: a row of the data-parallel moves
static_assert(LANES == 16, "group_max works on rows of 16 lanes");
constexpr int LIST = 52;

struct Entry {
    char *param;
    const char *grad;
    float *master;
    char *m, *v;
    uint16_t *scales;
    uint64_t count_types; // elements; type of the gradient in bits 48 on, of the parameters in bits 56 on
    float lr_decay;
    uint32_t key; // of the random bits
};
struct TensorList {
    Entry t[LIST];
    uint32_t first[LIST + 1]; // a tensor's tiles are [first[i], first[i + 1])
};
struct Step {
    const float *factor;
    const float *counted; // NULL, or 1 / c1 and 1 / c2 where the steps are counted on the device
    float lr, beta1, omb1, beta2, omb2, eps, inv_c1, inv_c2; // omb = 1 - beta, rounded from fp64
    int32_t tensors;
    uint32_t tiles;
};
static_assert(sizeof(TensorList) + sizeof(Step) <= 4096, "kernel arguments");

template <int CTRL> __device__ inline uint32_t dpp_u(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true); }

__device__ inline uint32_t group_max(uint32_t v)
{
    v = max(v, dpp_u<0xB1>(v));
    v = max(v, dpp_u<0x4E>(v));
    v = max(v, dpp_u<0x141>(v));
    return max(v, dpp_u<0x140>(v));
}

template <class T> __device__ inline void load8(const T *p, int left, float (&v)[EACH])
{
    constexpr int V = 16 / sizeof(T);
    if (left >= EACH) {
#pragma unroll
        for (int i = 0; i < EACH; i += V) {
            const auto x = load_vec<T, V>(p + i);
#pragma unroll
            for (int j = 0; j < V; ++j) v[i + j] = (float)x[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
}

template <class T> __device__ inline void store8(T *p, int left, const float (&v)[EACH])
{
    constexpr int V = 16 / sizeof(T);
    if (left >= EACH) {
#pragma unroll
        for (int i = 0; i < EACH; i += V) {
            float x[V];
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = v[i + j];
            store_vec<T, V>(p + i, x);
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}

__device__ inline void load8_of(int type, const char *base, int64_t at, int left, float (&v)[EACH])
{
    if (type == SLICEGCN_F32) load8(reinterpret_cast<const float *>(base) + at, left, v);
    else if (type == SLICEGCN_BF16) load8(reinterpret_cast<const bf16 *>(base) + at, left, v);
    else load8(reinterpret_cast<const f16 *>(base) + at, left, v);
}

__device__ inline void store8_of(int type, char *base, int64_t at, int left, const float (&v)[EACH])
{
    if (type == SLICEGCN_F32) store8(reinterpret_cast<float *>(base) + at, left, v);
    else if (type == SLICEGCN_BF16) store8(reinterpret_cast<bf16 *>(base) + at, left, v);
    else store8(reinterpret_cast<f16 *>(base) + at, left, v);
}

typedef uint32_t codes2 __attribute__((ext_vector_type(2)));
typedef uint32_t codes2_packed __attribute__((ext_vector_type(2), aligned(1)));

__device__ inline codes2 load_codes(const char *p, int left)
{
    if (left >= EACH) return *reinterpret_cast<const codes2_packed *>(p);
    codes2 c = {0u, 0u};
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (i < left) c[i / 4] |= (uint32_t)(uint8_t)p[i] << (i % 4 * 8);
    return c;
}

__device__ inline void store_codes(char *p, int left, codes2 c)
{
    if (left >= EACH) {
        *reinterpret_cast<codes2_packed *>(p) = c;
        return;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (i < left) p[i] = (char)(c[i / 4] >> (i % 4 * 8));
}

__device__ inline float power_of(uint32_t biased) { return __uint_as_float(biased << 23); }

__device__ inline void decode(codes2 c, uint32_t byte, float (&v)[EACH])
{
    const float scale = power_of(byte);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
        v[4 * w] = lo[0] * scale;
        v[4 * w + 1] = lo[1] * scale;
        v[4 * w + 2] = hi[0] * scale;
        v[4 * w + 3] = hi[1] * scale;
    }
}

// The codes of 8 values of a block, and the block's byte.  SHIFT: which half of the random words decides.  SQUARE: values >= 0 that are never stored as 0
// unless they are.
template <int SHIFT, bool SQUARE> __device__ inline codes2 encode(const float (&v)[EACH], const uint32_t (&noise)[EACH], uint32_t &byte)
{
#pragma clang fp contract(off)
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        most = max(most, b < 0x7f800000u ? b : 0u);
    }
    most = group_max(most) >> 23;
    byte = most > 8 ? most - 7 : 1u;
    const float to_grid = power_of(254u - byte), least = 0.015625f; // 2^-6, the smallest normal number of the grid: below it, it is that of the binade above
    float t[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const float x = fabsf(v[i]) * to_grid, lift = x < least ? least : 0.f;
        const uint32_t r = SHIFT ? noise[i] >> 16 : noise[i] & 0xffffu;
        t[i] = __uint_as_float((__float_as_uint(x + lift) + (r << 4)) & 0xfff00000u) - lift;
        if (SQUARE) t[i] = v[i] > 0.f && t[i] == 0.f ? 0.001953125f : t[i];
        if ((__float_as_uint(v[i]) & 0x7fffffffu) >= 0x7f800000u) t[i] = __uint_as_float(0x7fc00000u);
        t[i] = copysignf(t[i], v[i]);
    }
    codes2 c;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * w], t[4 * w + 1], 0, false);
        c[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[4 * w + 2], t[4 * w + 3], x, true);
    }
    return c;
}

// The instruction takes a subnormal number for 0, and an update of 1 would become one of sqrt(v) / eps: 10^10 with v = 10^-40 and eps = 10^-30.  So it is given v 2^64 below 2^-96.
// What it gives for all others is as before.  (v itself is 0 where g^2 is, below some 10^-23 |g|.)
__device__ inline float root(float v)
{
    const bool small = v < 0x1p-96f;
    return __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.f);
}

// One more step taken, where it is taken at all, and its corrections
__global__ void count_kernel(int32_t *counter, const float *factor, double beta1, double beta2)
{
    if (factor && !(*factor > 0.f)) return;
    const int32_t step = counter[0] < INT32_MAX ? counter[0] + 1 : counter[0];
    counter[0] = step;
    float *c = reinterpret_cast<float *>(counter);
    c[1] = (float)(1.0 / (1.0 - pow(beta1, (double)step)));
    c[2] = (float)(1.0 / (1.0 - pow(beta2, (double)step)));
}

template <int STATES> __global__ __launch_bounds__(THREADS) void adamw_kernel(const TensorList list, const Step s)
{
#pragma clang fp contract(off)
    const float f = s.factor ? *s.factor : 1.f;
    if (!(f > 0.f)) return;
    const float inv_c1 = s.counted ? s.counted[0] : s.inv_c1, inv_c2 = s.counted ? s.counted[1] : s.inv_c2;
    int at = 0;
    for (uint32_t tile = blockIdx.x; tile < s.tiles; tile += gridDim.x) {
        int hi = s.tensors; // the tensor that holds the tile: the last one that starts at or before it
        while (hi - at > 1) {
            const int mid = (at + hi) / 2;
            if (list.first[mid] <= tile) at = mid;
            else hi = mid;
        }
        const Entry &e = list.t[at];
        const int64_t count = (int64_t)(e.count_types & (((uint64_t)1 << 48) - 1)), i0 = (int64_t)(tile - list.first[at]) * TILE + threadIdx.x * EACH;
        const int grad_type = (int)(e.count_types >> 48) & 0xff, param_type = (int)(e.count_types >> 56);
        const int left = count - i0 < EACH ? (count > i0 ? (int)(count - i0) : 0) : EACH;
        float p[EACH], g[EACH], m[EACH], v[EACH];
        load8_of(grad_type, e.grad, i0, left, g);
        if (e.master) load8(e.master + i0, left, p);
        else load8_of(param_type, e.param, i0, left, p);
        if constexpr (STATES == 8) {
            const uint32_t bytes = left > 0 ? e.scales[i0 / BLOCK] : 0x0101u;
            decode(load_codes(e.m + i0, left), bytes & 0xffu, m);
            decode(load_codes(e.v + i0, left), bytes >> 8, v);
        } else {
            load8(reinterpret_cast<const float *>(e.m) + i0, left, m);
            load8(reinterpret_cast<const float *>(e.v) + i0, left, v);
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            g[i] = g[i] * f;
            m[i] = m[i] * s.beta1 + g[i] * s.omb1;
            v[i] = v[i] * s.beta2 + (g[i] * g[i]) * s.omb2;
            const float update = (m[i] * inv_c1) * __builtin_amdgcn_rcpf(root(v[i] * inv_c2) + s.eps);
            p[i] = p[i] - e.lr_decay * p[i] - s.lr * update;
        }
        if (e.master) store8(e.master + i0, left, p);
        store8_of(param_type, e.param, i0, left, p);
        if constexpr (STATES == 8) {
            uint32_t noise[EACH], bytes[2];
            const uint32_t x0 = (uint32_t)i0 * 0x9E3779B9u + e.key;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                uint32_t x = x0 + (uint32_t)i * 0x9E3779B9u;
                x ^= x >> 15;
                x *= 0xA54FF53Bu;
                noise[i] = x ^ (x >> 16);
            }
            // elements behind the last one are zeros, of which every value here is one
            const codes2 cm = encode<1, false>(m, noise, bytes[0]), cv = encode<0, true>(v, noise, bytes[1]);
            store_codes(e.m + i0, left, cm);
            store_codes(e.v + i0, left, cv);
            if (threadIdx.x % LANES == 0 && left > 0) e.scales[i0 / BLOCK] = (uint16_t)(bytes[0] | bytes[1] << 8);
        } else {
            store8(reinterpret_cast<float *>(e.m) + i0, left, m);
            store8(reinterpret_cast<float *>(e.v) + i0, left, v);
        }
    }
}

int check(const slicegcn_adam_tensor *ts, int32_t count, int32_t states, double lr, double beta1, double beta2, double eps, int32_t step)
{
    SG_REQUIRE(count >= 0 && (ts || count == 0), SLICEGCN_EINVAL, "adamw_step: NULL tensors, or count < 0");
    SG_REQUIRE(states == SLICEGCN_STATES_8 || states == SLICEGCN_STATES_32, SLICEGCN_EINVAL, "adamw_step: states of %d bits", states);
    SG_REQUIRE(step >= 1, SLICEGCN_EINVAL, "adamw_step: step must be >= 1");
    SG_REQUIRE(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0, SLICEGCN_EINVAL, "adamw_step: betas must lie in [0, 1)");
    // 1 / eps is a number of fp32 then, and an m of 0 moves nothing where v is 0 too
    SG_REQUIRE(std::isfinite((float)lr) && (float)eps >= FLT_MIN && std::isfinite((float)eps), SLICEGCN_EINVAL, "adamw_step: lr must be finite and eps at least 2^-126");
    for (int32_t i = 0; i < count; ++i) {
        const slicegcn_adam_tensor &t = ts[i];
        SG_REQUIRE(t.count >= 0 && t.count <= (int64_t)1 << 40, SLICEGCN_EINVAL, "adamw_step: tensor %d has %lld elements", i, (long long)t.count);
        SG_REQUIRE(known_type(t.param_type) && known_type(t.grad_type), SLICEGCN_EINVAL, "adamw_step: tensor %d: unknown type", i);
        SG_REQUIRE(std::isfinite(t.decay), SLICEGCN_EINVAL, "adamw_step: tensor %d: decay is not finite", i);
        SG_REQUIRE(!t.master || t.param_type != SLICEGCN_F32, SLICEGCN_EINVAL, "adamw_step: tensor %d: a master of fp32 parameters", i);
        if (t.count == 0) continue;
        SG_REQUIRE(t.param && t.grad && t.m && t.v && (t.scales || states == SLICEGCN_STATES_32), SLICEGCN_EINVAL, "adamw_step: tensor %d: NULL pointer", i);
        const auto on = [](const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; };
        SG_REQUIRE(aligned_for(t.param, t.param_type) && aligned_for(t.grad, t.grad_type) && on(t.master, 4) && on(t.scales, 2) &&
                       (states == SLICEGCN_STATES_8 || (on(t.m, 4) && on(t.v, 4))),
                   SLICEGCN_EINVAL, "adamw_step: tensor %d: misaligned", i);
    }
    return SLICEGCN_OK;
}

// counter: NULL where `step` says which step it is
int adamw(const slicegcn_adam_tensor *ts, int32_t count, int32_t states, double lr, double beta1, double beta2, double eps, int32_t step, int32_t *counter,
          const float *factor, uint64_t seed, void *stream)
{
    Step s{};
    s.factor = factor;
    s.counted = counter ? reinterpret_cast<const float *>(counter) + 1 : nullptr;
    s.lr = (float)lr;
    s.beta1 = (float)beta1;
    s.omb1 = (float)(1.0 - beta1);
    s.beta2 = (float)beta2;
    s.omb2 = (float)(1.0 - beta2);
    s.eps = (float)eps;
    s.inv_c1 = (float)(1.0 / (1.0 - pow(beta1, (double)step)));
    s.inv_c2 = (float)(1.0 / (1.0 - pow(beta2, (double)step)));
    const uint32_t key = (uint32_t)seed * 0x6A09E667u + (uint32_t)(seed >> 32) * 0xBB67AE85u;
    constexpr int64_t MOST_TILES = (int64_t)1 << 31;
    ProfScope prof(SLICEGCN_PROF_ADAMW, count, as_stream(stream));
    if (counter) {
        count_kernel<<<1, 1, 0, as_stream(stream)>>>(counter, factor, beta1, beta2);
        SG_LAUNCH_CHECK();
    }
    TensorList list;
    int64_t tiles = 0;
    int n = 0;
    auto flush = [&]() -> int {
        if (n == 0) return SLICEGCN_OK;
        list.first[n] = (uint32_t)tiles;
        s.tensors = n;
        s.tiles = (uint32_t)tiles;
        const unsigned blocks = (unsigned)(tiles < 4096 ? tiles : 4096);
        if (states == SLICEGCN_STATES_8) adamw_kernel<8><<<blocks, THREADS, 0, as_stream(stream)>>>(list, s);
        else adamw_kernel<32><<<blocks, THREADS, 0, as_stream(stream)>>>(list, s);
        SG_LAUNCH_CHECK();
        n = 0;
        tiles = 0;
        return SLICEGCN_OK;
    };
    for (int32_t i = 0; i < count; ++i) {
        const slicegcn_adam_tensor &t = ts[i];
        if (t.count == 0) continue;
        const int64_t want = (t.count + TILE - 1) / TILE;
        if (n == LIST || tiles + want > MOST_TILES)
            if (int rc = flush()) return rc;
        Entry &e = list.t[n];
        e.param = static_cast<char *>(t.param);
        e.grad = static_cast<const char *>(t.grad);
        e.master = t.master;
        e.m = static_cast<char *>(t.m);
        e.v = static_cast<char *>(t.v);
        e.scales = reinterpret_cast<uint16_t *>(t.scales);
        e.count_types = (uint64_t)t.count | (uint64_t)t.grad_type << 48 | (uint64_t)t.param_type << 56;
        e.lr_decay = (float)(lr * (double)t.decay);
        e.key = key + (uint32_t)i * 0x3C6EF373u;
        list.first[n++] = (uint32_t)tiles;
        tiles += want;
    }
    return flush();
}

} // namespace
} // namespace slicegcn

using namespace slicegcn;

extern "C" int slicegcn_adamw_step(const slicegcn_adam_tensor *ts, int32_t count, int32_t states, double lr, double beta1, double beta2, double eps,
                                   int32_t step, const float *factor, uint64_t seed, void *stream)
{
    if (int rc = check(ts, count, states, lr, beta1, beta2, eps, step)) return rc;
    return adamw(ts, count, states, lr, beta1, beta2, eps, step, nullptr, factor, seed, stream);
}

extern "C" int slicegcn_adamw_step_counted(const slicegcn_adam_tensor *ts, int32_t count, int32_t states, double lr, double beta1, double beta2, double eps,
                                           int32_t *counter, const float *factor, uint64_t seed, void *stream)
{
    if (int rc = check(ts, count, states, lr, beta1, beta2, eps, 1)) return rc;
    SG_REQUIRE(counter && (reinterpret_cast<uintptr_t>(counter) & 3u) == 0, SLICEGCN_EINVAL, "adamw_step_counted: NULL or misaligned counter");
    return adamw(ts, count, states, lr, beta1, beta2, eps, 1, counter, factor, seed, stream);
}
