// Norms before and after a block, fused with the block's gate and the residual, forward and backward.
//
//   p = post(y) * post_w + post_b;   h = residual * x + s * p;   u = pre(h) * pre_w + pre_b
//
// With yn, hn the normalised rows, ry, rh the factors 1 / sqrt(...) they were multiplied by, and means over a row's columns:
//   dun = du * pre_w;    dH = dh + rh * (dun - [mean dun] - hn * mean(dun * hn))          [..]: layer norm only
//   dx = residual * dH;  dgate = dH * p (times s (1 - s) through a sigmoid)
//   dyn = dH * s * post_w;  dy = ry * (dyn - [mean dyn] - yn * mean(dyn * yn))
//   dpre_w = sum du * hn;  dpre_b = sum du;  dpost_w = sum dH * s * yn;  dpost_b = sum dH * s     (sums over rows)
// A gate per column has dgate = post_w * sum dH * yn + post_b * sum dH, so that two sums per norm serve all parameters.
//
// A row lies in the registers of a group of lanes from its one read to its one write, and h is formed again in the backward pass instead of
// being read (it would have to be kept, and rounded): bound by bytes.  Lanes hold 8 elements of a row each, so that the backward pass has room for
// the parameters of its columns, the sums over its rows and the operands of the row after, which is what keeps the memory busy while
// a row's sums go round its lanes.  Counters: every kernel moves its operands once (2 % more where rows are no whole lines).
// Measured (a 4 GiB copy moves 6.2 TB/s): forward 169 343 rows of 256 fp32 columns 121 us, 5.7 TB/s; 16 384 of 4096 bf16 84 us, 6.4 TB/s.
// Backward 16 384 of 4096 bf16 150 us, 5.4 TB/s; 232 965 of 602 fp32 with layer norms and a sigmoid gate per element 870 us, 5.2 TB/s.
// Above 4096 columns a row takes 1024 threads of 128 registers each.  Forward: parameters are read again for every row and no row is requested ahead, fp32 rows
// 5.1 to 5.4 TB/s with RMS norms and 3.3 to 4.6 with layer norms or a gate per element, 16-bit rows 3.4 to 3.7 and 2.0 to 3.2.  Backward: 5.0 to 5.4
// TB/s with RMS norms and 3.0 to 4.6 with layer norms or a gate per element (sums over rows lie in LDS, in registers they spilled: 1.4 to 2.4).  Above 8192
// columns, where twice the elements do not fit the registers: forward 4.3 to 5.6 TB/s in fp32 and 3.8 to 4.4 in 16 bits with RMS norms, else 1.5 to 2.8; backward
// 1.5 to 2.9 with RMS norms, else 0.7 to 1.4.
#pragma once

#include "resnorm.h"

#include <cfloat>

namespace slicegcn {
namespace resnorm {

namespace {

template <int V> struct Lane { // K accesses of V columns; the last access of a row that is no multiple of V wide is moved left
    int32_t col;
    int skip; // leading columns that the access before it holds too
    bool on;
};

template <class T, int V, int K> struct Raw { typename VecOf<T, V>::type v[K]; }; // a lane's part of a row, as it lies in memory

// COUNTS: which columns count in sums is held as factors over all rows, or found out each time
template <class T, int V, int K, bool MULTI, bool FULL, bool COUNTS> struct Row {
    const Args &a;
    float *shared; // MULTI: [2][16][2]
    int lane, slot; // lane within the row, row within the workgroup
    int turn = 0;
    Lane<V> at[K];
    float counts[COUNTS ? K : 1][COUNTS ? V : 1]; // 1 where the column counts in the lane's sums, 0 where another lane holds it too or it lies past the end

    __device__ Row(const Args &args, float *sh) : a(args), shared(sh)
    {
        slot = threadIdx.x / a.lanes;
        lane = threadIdx.x - slot * a.lanes;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t c = (lane + k * a.lanes) * V;
            at[k].on = FULL || c < a.width;
            at[k].col = FULL ? c : min(c, a.width - V);
            at[k].skip = FULL ? 0 : c - at[k].col;
            if constexpr (COUNTS) {
#pragma unroll
                for (int j = 0; j < V; ++j) counts[k][j] = at[k].on && j >= at[k].skip ? 1.f : 0.f;
            }
        }
    }

    // sum of f(k, j) * g(k, j) over the lane's columns
    template <class F, class G> __device__ float lane_dot(F f, G g) const
    {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!COUNTS && !at[k].on) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (FULL) s = fmaf(f(k, j), g(k, j), s);
                else if constexpr (COUNTS) s = fmaf(f(k, j) * counts[k][j], g(k, j), s);
                else s = fmaf(j >= at[k].skip ? f(k, j) : 0.f, g(k, j), s);
            }
        }
        return s;
    }

    // Sum of squares.  A column that another lane counts is left out, not multiplied by 0: where it holds an infinity, that would be NaN.
    template <class F> __device__ float lane_squares(F f) const
    {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!COUNTS && !at[k].on) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v = f(k, j);
                if constexpr (COUNTS) v = counts[k][j] != 0.f ? v : 0.f;
                else if constexpr (!FULL) v = j >= at[k].skip ? v : 0.f;
                s = fmaf(v, v, s);
            }
        }
        return s;
    }

    template <class F> __device__ float lane_sum(F f) const
    {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!COUNTS && !at[k].on) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (FULL) s += f(k, j);
                else if constexpr (COUNTS) s = fmaf(f(k, j), counts[k][j], s);
                else s += j >= at[k].skip ? f(k, j) : 0.f;
            }
        }
        return s;
    }

    // N sums over the row's lanes, in every lane
    template <int N> __device__ void over_lanes(float (&s)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = group_sum(s[i], MULTI ? 64 : a.lanes);
        if (!MULTI) return;
        float *buf = shared + turn * 32; // written again two sums later, when every wavefront has read it
        turn ^= 1;
        const int wave = threadIdx.x / 64, waves = a.lanes / 64, first = slot * waves;
        if (threadIdx.x % 64 == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) buf[2 * wave + i] = s[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = 0.f;
        for (int w = 0; w < waves; ++w) {
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] += buf[2 * (first + w) + i];
        }
    }

    __device__ Raw<T, V, K> load(const RowPtr &p, int64_t row, bool there) const
    {
        Raw<T, V, K> r;
        const T *q = reinterpret_cast<const T *>(p.data) + row * p.ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (there && at[k].on) {
                r.v[k] = load_vec<T, V>(q + at[k].col);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) r.v[k][j] = (T)0.f;
            }
        }
        return r;
    }

    __device__ void store(const RowPtr &p, int64_t row, const float (&v)[K][V]) const
    {
        T *q = reinterpret_cast<T *>(p.data) + row * p.ld;
        if (a.past_cache) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (at[k].on) store_vec_past_cache<T, V>(q + at[k].col, v[k]);
            asm volatile(""); // keeps the two kinds of stores apart: made into one they would be plain ones
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (at[k].on) store_vec<T, V>(q + at[k].col, v[k]);
        }
    }

    // the lane's columns of a parameter, or `absent`
    __device__ void param(const float *p, float absent, float (&v)[K][V]) const
    {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (p) {
                const auto w = load_vec<float, V>(p + at[k].col);
#pragma unroll
                for (int j = 0; j < V; ++j) v[k][j] = w[j];
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[k][j] = absent;
            }
        }
    }

    template <class F> __device__ void each(F f) const
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) f(k, j);
    }

    // mean and 1 / sqrt(...) of a row
    __device__ void moments(const float (&v)[K][V], int kind, float *mean, float *factor)
    {
        float s[1];
        *mean = 0.f;
        if (kind == LAYER) {
            s[0] = lane_sum([&](int k, int j) { return v[k][j]; });
            over_lanes(s);
            *mean = s[0] * a.inv_width;
        }
        const float m = *mean;
        s[0] = lane_squares([&](int k, int j) { return v[k][j] - m; });
        over_lanes(s);
        *factor = rsqrtf(s[0] * a.inv_width + a.eps); // one operation, off by a unit in the last place at most
    }

    // s, the factor of p, from a gate
    __device__ float opened(float g) const { return a.sigmoid ? 1.f / (1.f + expf(-g)) : g; }

    // The same, and q times the slope s (1 - s) of a sigmoid.  With e = exp(-g), 1 - s is e s: formed as 1 - s, it would keep nothing of an s near 1.
    __device__ float opened(float g, float *q) const
    {
        if (!a.sigmoid) return g;
        const float e = expf(-g), s = 1.f / (1.f + e);
        *q *= fminf(e, FLT_MAX) * s * s; // an e of infinity has an s of 0
        return s;
    }
};

// Parameters of the lane's columns, held over all rows.  With a gate per column (or none) s * p is one product: yn * (s * post_w) + s * post_b.
// A workgroup of 1024 threads has registers for one row only: there the parameters are read again for every row, from the caches.
template <int V, int K> struct Held {
    float w[K][V], b[K][V], pre_w[K][V], pre_b[K][V];
    template <bool MATRIX, bool EXTRA, bool FWD, class R> __device__ void load(const R &r, const Args &a)
    {
        r.param(a.post_w, 1.f, w);
        if (EXTRA) r.param(a.post_b, 0.f, b);
        r.param(a.pre_w, 1.f, pre_w);
        if (EXTRA && FWD) r.param(a.pre_b, 0.f, pre_b);
        if (!MATRIX && a.gate_col) {
            float g[K][V];
            r.param(a.gate_col, 1.f, g);
            r.each([&](int k, int j) {
                const float s = r.opened(g[k][j]);
                w[k][j] *= s;
                if (EXTRA) b[k][j] *= s;
            });
        }
    }
};

// EXTRA: a layer norm or a bias anywhere
template <class T, int V, int K, bool MULTI, bool FULL, int THREADS, bool MATRIX, bool EXTRA>
__global__ __launch_bounds__(THREADS) void resnorm_fwd_kernel(const Args a)
{
    __shared__ float shared[MULTI ? 64 : 1];
    constexpr bool HOLD = THREADS < 1024, LOOP = HOLD && fwd_loops(MULTI, FULL, sizeof(T));
    Row<T, V, K, MULTI, FULL, LOOP && !MULTI> r(a, shared);
    Held<V, K> p;
    if (HOLD) p.template load<MATRIX, EXTRA, true>(r, a);
    const int rows = blockDim.x / a.lanes;
    const int64_t stride = (int64_t)gridDim.x * rows;
    Raw<T, V, K> next_x, next_y, next_g;
    auto request = [&](int64_t row) {
        const bool there = row < a.n;
        if (a.x.data) next_x = r.load(a.x, row, there);
        if (a.y.data) next_y = r.load(a.y, row, there);
        if (MATRIX) next_g = r.load(a.gate, row, there);
    };
    if (LOOP) request((int64_t)blockIdx.x * rows + r.slot);
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n; r0 += stride) {
        const int64_t row = r0 + r.slot;
        const bool there = row < a.n;
        float h[K][V], st[4] = {0.f, 1.f, 0.f, 1.f};
        if (!LOOP) request(row);
        if (!HOLD) p.template load<MATRIX, EXTRA, true>(r, a);
        const Raw<T, V, K> x = next_x, y = next_y, g = next_g;
        if (LOOP && r0 + stride < a.n) request(row + stride);
        if (a.x.data) r.each([&](int k, int j) { h[k][j] = a.residual * (float)x.v[k][j]; });
        else r.each([&](int k, int j) { h[k][j] = 0.f; });
        if (a.y.data) {
            float v[K][V];
            r.each([&](int k, int j) { v[k][j] = (float)y.v[k][j]; });
            if (a.post != NONE) {
                r.moments(v, EXTRA ? a.post : (int)SLICEGCN_NORM_RMS, &st[0], &st[1]);
                r.each([&](int k, int j) { v[k][j] = EXTRA ? (v[k][j] - st[0]) * st[1] : v[k][j] * st[1]; });
            }
            r.each([&](int k, int j) {
                if (MATRIX) {
                    const float q = EXTRA ? fmaf(v[k][j], p.w[k][j], p.b[k][j]) : v[k][j] * p.w[k][j];
                    h[k][j] = fmaf(r.opened((float)g.v[k][j]), q, h[k][j]);
                } else {
                    if (EXTRA) h[k][j] += p.b[k][j];
                    h[k][j] = fmaf(v[k][j], p.w[k][j], h[k][j]);
                }
            });
        }
        // rows in place: all of a row is read before any of it is written (a sum over the row sees to that too)
        if (MULTI && !FULL && !(a.y.data && a.post != NONE)) __syncthreads();
        if (a.h.data && there) r.store(a.h, row, h);
        if (a.u.data) {
            if (a.pre != NONE) {
                r.moments(h, EXTRA ? a.pre : (int)SLICEGCN_NORM_RMS, &st[2], &st[3]);
                r.each([&](int k, int j) {
                    h[k][j] = EXTRA ? fmaf((h[k][j] - st[2]) * st[3], p.pre_w[k][j], p.pre_b[k][j]) : h[k][j] * st[3] * p.pre_w[k][j];
                });
            }
            if (there) r.store(a.u, row, h);
        }
        if (a.stats && there && r.lane == 0) *reinterpret_cast<float4 *>(a.stats + 4 * row) = make_float4(st[0], st[1], st[2], st[3]);
    }
}

// The rows that the backward pass reads of one row: requested a row ahead
template <class T, int V, int K> struct Operands {
    Raw<T, V, K> x, y, g, dh, du;
    float4 st;
    template <bool MATRIX, class R> __device__ void request(const R &r, const Args &a, int64_t row, bool there)
    {
        if (a.x.data) x = r.load(a.x, row, there);
        if (a.y.data) y = r.load(a.y, row, there);
        if (MATRIX) g = r.load(a.gate, row, there);
        if (a.dh.data) dh = r.load(a.dh, row, there);
        if (a.du.data) du = r.load(a.du, row, there);
        st = there ? *reinterpret_cast<const float4 *>(a.stats + 4 * row) : make_float4(0.f, 1.f, 0.f, 1.f);
    }
};

template <class T, int V, int K, bool MULTI, bool FULL, int THREADS, bool MATRIX, bool EXTRA>
__global__ __launch_bounds__(THREADS) void resnorm_bwd_kernel(const Args a)
{
    __shared__ float shared[MULTI ? 64 : 1];
    // with a gate per element fp32 rows have no registers for the factors too: 232 965 rows of 602 with both 927 us, without the factors 855 (with a gate
    // per column 824 and 884; all before the sums over rows had their second level)
    Row<T, V, K, MULTI, FULL, !FULL && THREADS < 1024 && !(MATRIX && sizeof(T) == 4)> r(a, shared);
    // A workgroup of 1024 threads has registers for the parameters and a row ahead only without a gate per element, and in fp32 without layer norms and
    // biases.  TB/s at 8192 columns with / without: bf16 layer norms 4.1 / 2.9, with a gate per element 3.4 / 3.6; fp32 RMS norms 4.6 / 4.5, layer
    // norms 3.2 / 3.7.
    constexpr bool HOLD = THREADS < 1024 || (K * V == ELEMS && !MATRIX && (sizeof(T) == 2 || !EXTRA));
    Held<V, K> p;
    if (HOLD) p.template load<MATRIX, EXTRA, false>(r, a);
    const int rows = blockDim.x / a.lanes;
    const int64_t stride = (int64_t)gridDim.x * rows;
    // The sums over rows: in registers, added to places of the lane's own in LDS every FLUSH rows, so that long sums lose little (232 965 rows of 602
    // on 512 workgroups: off by 1.3e-7 of their size for 2.9e-7, in 2 % more time); where 1024 threads have no registers to spare, in LDS throughout.
    constexpr int FLUSH = 16, HELD_PLANES = EXTRA ? PLANES : PLANES / 2;
    constexpr bool IN_LDS = THREADS == 1024 && HELD_PLANES * K * V <= PLANES * ELEMS, FLUSHES = THREADS < 1024;
    __shared__ float own[IN_LDS || FLUSHES ? HELD_PLANES * K * THREADS * V : 1];
    float acc[IN_LDS ? 1 : PLANES][IN_LDS ? 1 : K][IN_LDS ? 1 : V] = {};
    const auto place = [&](int q, int k) { return own + (((EXTRA ? q : q / 2) * K + k) * THREADS + threadIdx.x) * V; };
    if constexpr (IN_LDS || FLUSHES) {
        const float zero[V] = {};
        for (int q = 0; q < PLANES; q += EXTRA ? 1 : 2)
#pragma unroll
            for (int k = 0; k < K; ++k) store_vec<float, V>(place(q, k), zero);
    }
    const auto flush = [&]() {
        if constexpr (FLUSHES) {
#pragma unroll
            for (int q = 0; q < PLANES; q += EXTRA ? 1 : 2)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const auto old = load_vec<float, V>(place(q, k));
                    float sum[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        sum[j] = old[j] + acc[q][k][j];
                        acc[q][k][j] = 0.f;
                    }
                    store_vec<float, V>(place(q, k), sum);
                }
        }
    };
    // plane q += f(k, j) * g(k, j)
    const auto add = [&](int q, auto f, auto g) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if constexpr (IN_LDS) {
                const auto old = load_vec<float, V>(place(q, k));
                float sum[V];
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] = fmaf(f(k, j), g(k, j), old[j]);
                store_vec<float, V>(place(q, k), sum);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) acc[q][k][j] = fmaf(f(k, j), g(k, j), acc[q][k][j]);
            }
        }
    };
    const auto one = [](int, int) { return 1.f; };
    Operands<T, V, K> next;
    if (HOLD && (int64_t)blockIdx.x * rows < a.n) next.template request<MATRIX>(r, a, (int64_t)blockIdx.x * rows + r.slot, (int64_t)blockIdx.x * rows + r.slot < a.n);
    int since = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n; r0 += stride) {
        const int64_t row = r0 + r.slot;
        const bool there = row < a.n;
        if (FLUSHES && ++since == FLUSH) {
            flush();
            since = 0;
        }
        if (!HOLD) {
            next.template request<MATRIX>(r, a, row, there);
            p.template load<MATRIX, EXTRA, false>(r, a);
        }
        const Operands<T, V, K> o = next;
        if (HOLD && r0 + stride < a.n) next.template request<MATRIX>(r, a, row + stride, row + stride < a.n);
        float h[K][V], yn[K][V], dH[K][V], q[K][V], s[K][V];
        if (a.x.data) r.each([&](int k, int j) { h[k][j] = a.residual * (float)o.x.v[k][j]; });
        else r.each([&](int k, int j) { h[k][j] = 0.f; });
        if (a.y.data) { // h again, from what it was formed of
            r.each([&](int k, int j) {
                yn[k][j] = EXTRA ? ((float)o.y.v[k][j] - o.st.x) * o.st.y : (float)o.y.v[k][j] * o.st.y;
                if (MATRIX) {
                    const float v = EXTRA ? fmaf(yn[k][j], p.w[k][j], p.b[k][j]) : yn[k][j] * p.w[k][j];
                    q[k][j] = v;
                    s[k][j] = r.opened((float)o.g.v[k][j], &q[k][j]);
                    h[k][j] = fmaf(s[k][j], v, h[k][j]);
                } else {
                    if (EXTRA) h[k][j] += p.b[k][j];
                    h[k][j] = fmaf(yn[k][j], p.w[k][j], h[k][j]);
                }
            });
        }
        if (a.dh.data) r.each([&](int k, int j) { dH[k][j] = (float)o.dh.v[k][j]; });
        else r.each([&](int k, int j) { dH[k][j] = 0.f; });
        if (a.du.data) {
            if (a.pre == NONE) {
                r.each([&](int k, int j) { dH[k][j] += (float)o.du.v[k][j]; });
            } else {
                float d[K][V];
                r.each([&](int k, int j) { h[k][j] = EXTRA ? (h[k][j] - o.st.z) * o.st.w : h[k][j] * o.st.w; }); // hn
                const auto du = [&](int k, int j) { return (float)o.du.v[k][j]; };
                if (a.planes & 1) add(0, du, [&](int k, int j) { return h[k][j]; });
                if (EXTRA && (a.planes & 2)) add(1, du, one);
                r.each([&](int k, int j) { d[k][j] = (float)o.du.v[k][j] * p.pre_w[k][j]; });
                float c[2] = {r.lane_dot([&](int k, int j) { return d[k][j]; }, [&](int k, int j) { return h[k][j]; }), 0.f};
                if (EXTRA && a.pre == LAYER) {
                    c[1] = r.lane_sum([&](int k, int j) { return d[k][j]; });
                    r.over_lanes(c);
                } else {
                    float first[1] = {c[0]};
                    r.over_lanes(first);
                    c[0] = first[0];
                }
                c[0] *= a.inv_width;
                c[1] *= a.inv_width;
                r.each([&](int k, int j) { dH[k][j] = fmaf(o.st.w, fmaf(-h[k][j], c[0], EXTRA ? d[k][j] - c[1] : d[k][j]), dH[k][j]); });
            }
        }
        if (MULTI && !FULL && !(a.du.data && a.pre != NONE)) __syncthreads(); // rows in place, as in the forward pass
        if (a.dx.data && there) {
            r.each([&](int k, int j) { h[k][j] = a.residual * dH[k][j]; });
            r.store(a.dx, row, h);
        }
        if (!a.y.data) continue;
        if (MATRIX) {
            if (a.dgate.data && there) {
                r.each([&](int k, int j) { q[k][j] *= dH[k][j]; });
                r.store(a.dgate, row, q);
            }
            r.each([&](int k, int j) { dH[k][j] *= s[k][j]; });
        }
        const auto dp = [&](int k, int j) { return dH[k][j]; };
        if (a.planes & 4) add(2, dp, [&](int k, int j) { return yn[k][j]; });
        if (EXTRA && (a.planes & 8)) add(3, dp, one);
        if (!a.dy.data) continue;
        r.each([&](int k, int j) { dH[k][j] *= p.w[k][j]; });
        if (a.post != NONE) {
            float d[2] = {r.lane_dot([&](int k, int j) { return dH[k][j]; }, [&](int k, int j) { return yn[k][j]; }), 0.f};
            if (EXTRA && a.post == LAYER) {
                d[1] = r.lane_sum([&](int k, int j) { return dH[k][j]; });
                r.over_lanes(d);
            } else {
                float first[1] = {d[0]};
                r.over_lanes(first);
                d[0] = first[0];
            }
            d[0] *= a.inv_width;
            d[1] *= a.inv_width;
            r.each([&](int k, int j) { dH[k][j] = o.st.y * fmaf(-yn[k][j], d[0], EXTRA ? dH[k][j] - d[1] : dH[k][j]); });
        }
        if (there) r.store(a.dy, row, dH);
    }
    if (!a.planes) return;
    flush();
    // the workgroup's sums: over the rows it holds beside each other, in order
    float *out = a.partial + (int64_t)blockIdx.x * PLANES * a.width;
    if (rows == 1) {
#pragma unroll
        for (int q = 0; q < PLANES; q += EXTRA ? 1 : 2) {
            if (!(a.planes >> q & 1)) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!r.at[k].on) continue;
                float *to = out + q * a.width + r.at[k].col;
                if constexpr (IN_LDS || FLUSHES) *reinterpret_cast<typename VecOf<float, V>::packed *>(to) = load_vec<float, V>(place(q, k));
                else store_vec<float, V>(to, acc[q][k]);
            }
        }
        return;
    }
    if constexpr (THREADS <= 256) {
        __syncthreads();
        for (int q = 0; q < PLANES; q += EXTRA ? 1 : 2) {
            if (!(a.planes >> q & 1)) continue;
            // column c lies in access c / V of its row, that is in access k of lane l (where the last access was moved left, in its first columns too)
            for (int c = threadIdx.x; c < a.width; c += blockDim.x) {
                const int last = (a.width + V - 1) / V - 1, access = min(c / V, last), k = access / a.lanes, l = access - k * a.lanes;
                const int j = access == last ? c - (a.width - V) : c - access * V;
                const float *from = own + (((EXTRA ? q : q / 2) * K + k) * THREADS + l) * V + j;
                float sum = 0.f;
#pragma unroll 8
                for (int i = 0; i < rows; ++i) sum += from[i * a.lanes * V];
                out[q * a.width + c] = sum;
            }
        }
    }
}

template <bool BWD, class T, int V, int K, bool MULTI, bool FULL, int THREADS> void launch_kernel(const Args &a, int64_t blocks, int threads, hipStream_t s)
{
    with_flag(a.gate.data != nullptr, [&](auto matrix) {
        with_flag(a.post == LAYER || a.pre == LAYER || a.post_b || a.pre_b, [&](auto extra) {
            constexpr bool MATRIX = decltype(matrix)::value, EXTRA = decltype(extra)::value;
            if constexpr (BWD) resnorm_bwd_kernel<T, V, K, MULTI, FULL, THREADS, MATRIX, EXTRA><<<(unsigned)blocks, threads, 0, s>>>(a);
            else resnorm_fwd_kernel<T, V, K, MULTI, FULL, THREADS, MATRIX, EXTRA><<<(unsigned)blocks, threads, 0, s>>>(a);
        });
    });
}

// THREADS of the kernels: as many as a workgroup has, at most
template <bool BWD, class T, int V, int K> void launch_lanes(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream)
{
    const int threads = s.threads();
    if constexpr (V == 1) { // rows narrower than an access
        launch_kernel<BWD, T, V, K, false, false, 256>(a, blocks, threads, stream);
    } else if constexpr (K * V > ELEMS) { // the widest rows
        launch_kernel<BWD, T, V, K, true, false, 1024>(a, blocks, threads, stream);
    } else if (s.lanes <= 64) {
        if (s.full(a.width, V)) launch_kernel<BWD, T, V, K, false, true, 256>(a, blocks, threads, stream);
        else launch_kernel<BWD, T, V, K, false, false, 256>(a, blocks, threads, stream);
    } else if constexpr (K * V == ELEMS) { // rows with fewer elements a lane take fewer lanes
        if (s.lanes <= 256) launch_kernel<BWD, T, V, K, true, false, 256>(a, blocks, threads, stream);
        else if (s.lanes <= 512) launch_kernel<BWD, T, V, K, true, false, 512>(a, blocks, threads, stream);
        else launch_kernel<BWD, T, V, K, true, false, 1024>(a, blocks, threads, stream);
    }
}

template <bool BWD, class T> void launch_type(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream)
{
    constexpr int V = 16 / (int)sizeof(T);
    if (a.width < V) return launch_lanes<BWD, T, 1, 1>(a, s, blocks, stream);
    switch (s.accesses) {
    case 1: return launch_lanes<BWD, T, V, 1>(a, s, blocks, stream);
    case 2: return launch_lanes<BWD, T, V, 2>(a, s, blocks, stream);
    default:
        if constexpr (V == 4) {
            if (s.accesses == 3) return launch_lanes<BWD, T, V, 3>(a, s, blocks, stream);
            return launch_lanes<BWD, T, V, 4>(a, s, blocks, stream);
        }
    }
}

} // namespace

template <class T> void launch_fwd(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream) { launch_type<false, T>(a, s, blocks, stream); }
template <class T> void launch_bwd(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream) { launch_type<true, T>(a, s, blocks, stream); }

} // namespace resnorm
} // namespace slicegcn
