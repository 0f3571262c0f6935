// Group norm with an activation over channel-last grids, forward and backward.
//
// A sample's group is normalised with its own mean and variance,
//     xh = (x - mean) rstd,   y = act(gamma xh + beta),
// and with g = d_y act'(gamma xh + beta) the backward is
//     d_gamma = sum g xh,   d_beta = sum g,
//     d_x = rstd (gamma g - (S1 + xh S2) / n),   S1 = sum over the group of gamma g,   S2 of gamma g xh.
//
// What bounds it: memory.  A sum over the whole group stands between reading a value and using it.  A small sample (32 Ki values in slots of
// four channels, 16 Ki in slots of eight or one; see `hold`) stays in the registers of one workgroup meanwhile (one launch).  Larger ones
// are passed over twice: a pass that sums (forward: x; backward: x
// and d_y), a small kernel that joins the workgroups' sums, and a pass that writes, from the end back to the start: what the first
// pass read last is still in the 256 MB of Infinity Cache (160^3 x 32 in fp32, all kernels of a training step: 808 us, from the
// start 832; of planes in bf16 both 167).  Measured there: 117, 179, 214 and 285 us for 0.5, 1.0, 1.0 and 1.6 GB (4.5 to 5.9 TB/s; a copy of 2 GB 4.95), 24 planes
// of 256^2 x 32 in bf16 24, 34, 47 and 52 us for 0.1, 0.2, 0.2 and 0.3 GB (a copy of 128 MB, which the cache holds, 8.5).  In all passes a thread keeps to one
// slot of V neighbouring channels (16 bytes where channels and
// alignment allow), so a channel's parameters and sums stay in its registers, and neighbouring lanes read neighbouring bytes.  Slots of one channel cost
// little: 30 channels, which are not divisible by four, take 0.98 (fp32) and 0.97 (bf16) of the forward's time with 32, and 1.01 and 1.04 of the backward's.
//
// Sums: a thread sums differences to the first value that it sees, in fp32 (a mean far from zero does not cancel the
// variance); threads are joined as (count, mean, sum of squared differences), workgroups in fp64 in a fixed order, so that
// results do not change from call to call.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "lp_kernels.h"

namespace lp {

namespace {

constexpr int kThreads = 256;
template <int V> constexpr int kUnroll = V == 8 ? 2 : V == 1 ? 8 : 4;   // rows a thread has in flight
constexpr long long kMaxGrid = 1 << 20;  // workgroups of a launch; items beyond are taken in turn
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

struct NormDev {
    long long N, P;
    int C, G, Cg;
    long long xs, ys;                   // elements from position to position
    const float *gamma, *beta, *occ;
    float eps;
    int act;
    int slots, zblocks, rows;           // C / V; blocks of kThreads slots; positions a workgroup takes at a time
    int chunks;                         // items of a sample
    long long chunk;                    // positions of an item
};

using f32x2 = float __attribute__((ext_vector_type(2)));
using f32x4 = float __attribute__((ext_vector_type(4)));

template <class T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }
__device__ __forceinline__ float to_f32(_Float16 v) { return (float)v; }

template <class T, int V>
__device__ __forceinline__ void load(const T* p, Pack<T, V>& out)
{
    out = *reinterpret_cast<const Pack<T, V>*>(p);
}

template <class T, int V>
__device__ __forceinline__ void store(T* p, const float (&in)[V])
{
    Pack<T, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = (T)in[j];   // round to nearest even, once
    *reinterpret_cast<Pack<T, V>*>(p) = q;
}

// 1 / (1 + exp(-z)) from the hardware's exponential and reciprocal (a few units in the last place)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The normal distribution's integral up to z and its density.  For |z| < 1 the integral is 1/2 + z P(z^2), elsewhere the tail beyond
// |z| is t Q(t) exp(-z^2 / 2), t = 1 / (1 + 0.35 |z|) (0 at infinity, where t Q(t) goes like 1 / |z| as the tail does).  P and Q are fits
// of least largest relative error to the error function and its scaled complement in 64 bits, of 4.1e-8 and 1.1e-7.  With fp32 rounding, which
// enters the exponential's argument as 1.2e-7 z^2: relative error of the integral 4e-7 at z = -1, 1.4e-6 at -5, 5.2e-6 at -10.  The value and
// slope of the GELU are off by 2.3e-8 and 2.6e-8 (root mean square over a normal distribution), by the formula in fp32 torch by 2.5e-8 and 2.7e-8.
// (One polynomial for all z would be shorter and 4.4e-8 off in the slope.)
__device__ __forceinline__ void normal(float z, float& integral, float& density)
{
    const float a = fabsf(z), s = z * z, e = __builtin_amdgcn_exp2f(s * -0.72134752f), t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
    float tail = fmaf(t, 0.0431161788f, -0.109335177f);
    tail = fmaf(t, tail, 0.0433747092f);
    tail = fmaf(t, tail, 0.0312121292f);
    tail = fmaf(t, tail, 0.0901153928f);
    tail = fmaf(t, tail, 0.122394714f);
    tail = fmaf(t, tail, 0.139633358f);
    tail = fmaf(t, tail, 0.13962978f);
    tail *= t * e;
    float near = fmaf(s, 9.42352438e-05f, -0.0011693537f);
    near = fmaf(s, near, 0.00996719686f);
    near = fmaf(s, near, -0.0664895827f);
    near = fmaf(s, near, 0.398942264f);
    near = fmaf(z, near, 0.5f);
    asm("" : "+v"(near), "+v"(tail));   // (both are computed: branches around them took 24 registers more, of all activations' kernels)
    integral = a < 1.0f ? near : z < 0.0f ? tail : 1.0f - tail;
    density = e * kInvSqrt2Pi;
}

template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if (ACT == LP_ACT_RELU) return z < 0.0f ? 0.0f : z;   // (a NaN stays one)
    if (ACT == LP_ACT_SILU) return z * sigmoid(z);
    if (ACT == LP_ACT_GELU) {
        float i, d;
        normal(z, i, d);
        return z * i;
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z)
{
    if (ACT == LP_ACT_RELU) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    if (ACT == LP_ACT_SILU) {
        const float s = sigmoid(z);
        return fmaf(z * s, 1.0f - s, s);
    }
    if (ACT == LP_ACT_GELU) {
        float i, d;
        normal(z, i, d);
        return fmaf(z, d, i);
    }
    return 1.0f;
}

// Calls f with the activation as a constant: the choice stands outside the loops.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
        case LP_ACT_RELU: f(std::integral_constant<int, LP_ACT_RELU>()); break;
        case LP_ACT_SILU: f(std::integral_constant<int, LP_ACT_SILU>()); break;
        case LP_ACT_GELU: f(std::integral_constant<int, LP_ACT_GELU>()); break;
        default: f(std::integral_constant<int, LP_ACT_NONE>());
    }
}

// Where a thread stands: its slot of channels and its row among the positions a workgroup takes at a time.
struct Place {
    int slot, row;
    bool in;
};
__device__ __forceinline__ Place place(const NormDev& d)
{
    Place p;
    if (d.zblocks == 1) {
        p.row = threadIdx.x / d.slots;
        p.slot = threadIdx.x - p.row * d.slots;
        p.in = p.row < d.rows;
    } else {
        p.row = 0;
        p.slot = blockIdx.y * kThreads + threadIdx.x;
        p.in = p.slot < d.slots;
    }
    return p;
}

// Calls ld, then use, for the thread's positions of an item, U at a time: first all loads, then all of the rest.
template <int U, class Load, class Use>
__device__ __forceinline__ void sweep(const NormDev& d, long long first, long long end, int row, Load&& ld, Use&& use)
{
    for (long long p = first + row; p < end; p += (long long)U * d.rows) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long q = p + (long long)u * d.rows;
            ld(u, q, q < end);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long q = p + (long long)u * d.rows;
            use(u, q, q < end);
        }
    }
}

// A channel's parameters, for the V channels of a thread's slot.
template <int V>
struct Slot {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ void parameters(const NormDev& d, int slot)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            gamma[j] = d.gamma ? d.gamma[slot * V + j] : 1.0f;
            beta[j] = d.beta ? d.beta[slot * V + j] : 0.0f;
        }
    }
    // stats: [groups][2] of the sample
    __device__ __forceinline__ void statistics(const NormDev& d, int slot, const float* stats)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int g = (slot * V + j) / d.Cg;
            mean[j] = stats[2 * g];
            rstd[j] = stats[2 * g + 1];
        }
    }
};

// The sums of all threads of a slot, joined at row 0, lane by lane of a wave where a wave's rows are whole (then a wave counts as one
// row), then as a tree over the rows through LDS (2 V + 1 values a thread).  `join_two(count, a, b, other's ...)`.
template <int V, int THREADS, class F>
__device__ __forceinline__ void fold_rows(const NormDev& d, const Place& at, float& count, float (&a)[V], float (&b)[V], float* lds, F&& join_two)
{
    int all_rows = d.rows, row = at.row, step = d.slots;
    bool in = at.in;
    if (d.slots < 64 && (d.slots & (d.slots - 1)) == 0) {
        for (int o = 32; o >= d.slots; o >>= 1) {
            const float nb = __shfl_xor(count, o);
            float ab[V], bb[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ab[j] = __shfl_xor(a[j], o);
                bb[j] = __shfl_xor(b[j], o);
            }
            join_two(count, a, b, nb, ab, bb);
        }
        all_rows = THREADS / 64;
        row = threadIdx.x >> 6;
        step = 64;
        in = (int)(threadIdx.x & 63) < d.slots;
    }
    for (int rows = all_rows; rows > 1;) {
        const int half = (rows + 1) / 2;
        __syncthreads();
        if (in && row >= half && row < rows) {
            lds[threadIdx.x] = count;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                lds[(1 + j) * THREADS + threadIdx.x] = a[j];
                lds[(1 + V + j) * THREADS + threadIdx.x] = b[j];
            }
        }
        __syncthreads();
        if (in && row + half < rows) {
            const int o = threadIdx.x + half * step;
            float ab[V], bb[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ab[j] = lds[(1 + j) * THREADS + o];
                bb[j] = lds[(1 + V + j) * THREADS + o];
            }
            join_two(count, a, b, lds[o], ab, bb);
        }
        rows = half;
    }
}

template <int V, int THREADS>
__device__ __forceinline__ void join_rows(const NormDev& d, const Place& at, float& count, float (&mean)[V], float (&m2)[V], float* lds)
{
    fold_rows<V, THREADS>(d, at, count, mean, m2, lds, [](float& n, float (&m)[V], float (&q)[V], float nb, const float (&mb)[V], const float (&qb)[V]) {
        // (count, mean, sum of squared differences) of a joined with those of b
        const float total = n + nb, w = nb > 0.0f ? nb / total : 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float delta = mb[j] - m[j];
            if (nb > 0.0f) {
                q[j] = n > 0.0f ? q[j] + qb[j] + delta * delta * n * w : qb[j];
                m[j] = n > 0.0f ? m[j] + delta * w : mb[j];
            }
        }
        n = total;
    });
}

// The same for plain sums.
template <int V, int THREADS>
__device__ __forceinline__ void add_rows(const NormDev& d, const Place& at, float& count, float (&a)[V], float (&b)[V], float* lds)
{
    fold_rows<V, THREADS>(d, at, count, a, b, lds, [](float& n, float (&x)[V], float (&y)[V], float nb, const float (&xb)[V], const float (&yb)[V]) {
        n += nb;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[j] += xb[j];
            y[j] += yb[j];
        }
    });
}

// Sums of differences to a first value, and what they say of mean and m2.
template <int V>
struct Sums {
    float shift[V], s1[V], s2[V], count = 0.0f;
    __device__ Sums()
    {
#pragma unroll
        for (int j = 0; j < V; ++j) shift[j] = s1[j] = s2[j] = 0.0f;
    }
    template <class T>
    __device__ __forceinline__ void add(const Pack<T, V>& v)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float value = to_f32(v.v[j]);
            if (count == 0.0f) shift[j] = value;
            const float t = value - shift[j];
            s1[j] += t;
            s2[j] = fmaf(t, t, s2[j]);
        }
        count += 1.0f;
    }
    __device__ __forceinline__ void close(float (&mean)[V], float (&m2)[V]) const
    {
        const float inv = count > 0.0f ? 1.0f / count : 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float m = s1[j] * inv, v = s2[j] - s1[j] * m;
            mean[j] = shift[j] + m;
            m2[j] = v < 0.0f ? 0.0f : v;   // (a NaN stays one)
        }
    }
};

__device__ __forceinline__ void statistics_of(double n, double sum, double squares, float eps, float& mean, float& rstd)
{
    mean = rstd = 0.0f;
    if (n > 0.0) {
        const double m = sum / n;
        double var = squares / n - m * m;
        if (var < 0.0) var = 0.0;
        mean = (float)m;
        rstd = (float)(1.0 / sqrt(var + (double)eps));
    }
}

__device__ __forceinline__ double wave_sum(double v)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// ---- a sample in the registers of one workgroup ------------------------------------------------------------------

constexpr int kSmallThreads = 1024;
template <int V> constexpr int kHeld = V == 8 ? 2 : V == 4 ? 8 : 16;   // rows of a thread, at most

// One workgroup a sample, whose values stay in registers between the sums and the results: x is read once.
template <class TX, class TY, int V, bool MASK>
__global__ __launch_bounds__(kSmallThreads) void norm_small_kernel(NormDev d, const TX* x, TY* y, float* stats)
{
    __shared__ float lds[(2 * V + 1) * kSmallThreads];
    __shared__ float group_stats[2 * kSmallThreads];
    const Place at = place(d);
    const long long n = blockIdx.x;
    const TX* base = x + (size_t)(n * d.P) * d.xs + at.slot * V;
    const float* occ = MASK ? d.occ + n * d.P : nullptr;
    Pack<TX, V> v[kHeld<V>];
    bool on[kHeld<V>];
    Slot<V> slot;
#pragma unroll
    for (int k = 0; k < kHeld<V>; ++k) {
        const long long p = at.row + (long long)k * d.rows;
        on[k] = at.in && p < d.P && (!MASK || occ[p] > 0.0f);
        if (on[k]) load<TX, V>(base + p * d.xs, v[k]);
    }
    if (at.in) slot.parameters(d, at.slot);
    Sums<V> sums;
#pragma unroll
    for (int k = 0; k < kHeld<V>; ++k)
        if (on[k]) sums.add(v[k]);
    float count = sums.count, mean[V], m2[V];
    sums.close(mean, m2);
    join_rows<V, kSmallThreads>(d, at, count, mean, m2, lds);
    __syncthreads();
    if (at.in && at.row == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = at.slot * V + j;
            lds[3 * c] = count;
            lds[3 * c + 1] = mean[j];
            lds[3 * c + 2] = m2[j];
        }
    }
    __syncthreads();
    for (int g = threadIdx.x >> 6; g < d.G; g += kSmallThreads / 64) {
        double cnt = 0.0, sum = 0.0, sq = 0.0;
        for (int c = threadIdx.x & 63; c < d.Cg; c += 64) {
            const float* q = lds + 3 * (g * d.Cg + c);
            const double m = q[1];
            cnt += q[0];
            sum += (double)q[0] * m;
            sq += (double)q[2] + (double)q[0] * m * m;
        }
        cnt = wave_sum(cnt);
        sum = wave_sum(sum);
        sq = wave_sum(sq);
        if ((threadIdx.x & 63) == 0) {
            float mu, rstd;
            statistics_of(cnt, sum, sq, d.eps, mu, rstd);
            group_stats[2 * g] = mu;
            group_stats[2 * g + 1] = rstd;
            if (stats) {
                stats[(n * d.G + g) * 2] = mu;
                stats[(n * d.G + g) * 2 + 1] = rstd;
            }
        }
    }
    __syncthreads();
    if (!at.in) return;
    slot.statistics(d, at.slot, group_stats);
    TY* out = y + (size_t)(n * d.P) * d.ys + at.slot * V;
    with_act(d.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < kHeld<V>; ++k) {
            const long long p = at.row + (long long)k * d.rows;
            if (p >= d.P) continue;
            float r[V];
#pragma unroll
            for (int j = 0; j < V; ++j)
                r[j] = on[k] ? activate<decltype(act)::value>(fmaf((to_f32(v[k].v[j]) - slot.mean[j]) * slot.rstd[j], slot.gamma[j], slot.beta[j])) : 0.0f;
            store<TY, V>(out + p * d.ys, r);
        }
    });
}

// The same for the backward.  chan [n][C][2]: the samples' sums for the parameters; with a single sample they are added here.
template <class TX, class TY, int V, bool MASK>
__global__ __launch_bounds__(kSmallThreads) void norm_small_grad_kernel(NormDev d, const TX* x, const TY* dy, TX* dx, const float* __restrict__ stats,
                                                                        double* __restrict__ chan, float* d_gamma, float* d_beta)
{
    __shared__ float lds[(2 * V + 1) * kSmallThreads];
    __shared__ float means[2 * kSmallThreads];
    const Place at = place(d);
    const long long n = blockIdx.x;
    const TX* base = x + (size_t)(n * d.P) * d.xs + at.slot * V;
    const TY* up = dy + (size_t)(n * d.P) * d.ys + at.slot * V;
    const float* occ = MASK ? d.occ + n * d.P : nullptr;
    Pack<TX, V> v[kHeld<V>];
    Pack<TY, V> w[kHeld<V>];
    bool on[kHeld<V>];
    Slot<V> slot;
#pragma unroll
    for (int k = 0; k < kHeld<V>; ++k) {
        const long long p = at.row + (long long)k * d.rows;
        on[k] = at.in && p < d.P && (!MASK || occ[p] > 0.0f);
        if (on[k]) {
            load<TX, V>(base + p * d.xs, v[k]);
            load<TY, V>(up + p * d.ys, w[k]);
        }
    }
    if (at.in) {
        slot.parameters(d, at.slot);
        slot.statistics(d, at.slot, stats + n * d.G * 2);
    }
    float sg[V], sx[V], count = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) sg[j] = sx[j] = 0.0f;
    with_act(d.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < kHeld<V>; ++k) {
            if (!on[k]) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (to_f32(v[k].v[j]) - slot.mean[j]) * slot.rstd[j];
                const float g = to_f32(w[k].v[j]) * slope<decltype(act)::value>(fmaf(xh, slot.gamma[j], slot.beta[j]));
                sg[j] += g;
                sx[j] = fmaf(g, xh, sx[j]);
            }
            count += 1.0f;
        }
    });
    add_rows<V, kSmallThreads>(d, at, count, sg, sx, lds);
    __syncthreads();
    if (at.in && at.row == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = at.slot * V + j;
            lds[3 * c] = count;
            lds[3 * c + 1] = sg[j];
            lds[3 * c + 2] = sx[j];
            if (d.N > 1) {
                chan[(n * d.C + c) * 2] = sg[j];
                chan[(n * d.C + c) * 2 + 1] = sx[j];
            } else {
                if (d_beta) d_beta[c] += sg[j];
                if (d_gamma) d_gamma[c] += sx[j];
            }
        }
    }
    __syncthreads();
    for (int g = threadIdx.x >> 6; g < d.G; g += kSmallThreads / 64) {
        double cnt = 0.0, s1 = 0.0, s2 = 0.0;
        for (int j = threadIdx.x & 63; j < d.Cg; j += 64) {
            const int c = g * d.Cg + j;
            const double gamma = d.gamma ? d.gamma[c] : 1.0f;
            cnt += lds[3 * c];
            s1 += gamma * lds[3 * c + 1];
            s2 += gamma * lds[3 * c + 2];
        }
        cnt = wave_sum(cnt);
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if ((threadIdx.x & 63) == 0) {
            means[2 * g] = cnt > 0.0 ? (float)(s1 / cnt) : 0.0f;
            means[2 * g + 1] = cnt > 0.0 ? (float)(s2 / cnt) : 0.0f;
        }
    }
    __syncthreads();
    if (!at.in || !dx) return;
    float m1[V], mx[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int g = (at.slot * V + j) / d.Cg;
        m1[j] = means[2 * g];
        mx[j] = means[2 * g + 1];
    }
    TX* out = dx + (size_t)(n * d.P) * d.xs + at.slot * V;
    with_act(d.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < kHeld<V>; ++k) {
            const long long p = at.row + (long long)k * d.rows;
            if (p >= d.P) continue;
            float r[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                r[j] = 0.0f;
                if (on[k]) {
                    const float xh = (to_f32(v[k].v[j]) - slot.mean[j]) * slot.rstd[j];
                    const float g = to_f32(w[k].v[j]) * slope<decltype(act)::value>(fmaf(xh, slot.gamma[j], slot.beta[j]));
                    r[j] = slot.rstd[j] * (fmaf(slot.gamma[j], g, -m1[j]) - xh * mx[j]);
                }
            }
            store<TX, V>(out + p * d.xs, r);
        }
    });
}

// ---- in two passes ---------------------------------------------------------------------------------------------

// Pass 1 of the forward: (count, mean, m2) of every channel of every item -> part[((n C + c) chunks + chunk) 4].
template <class TX, int V, bool MASK>
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(NormDev d, const TX* __restrict__ x, f32x4* __restrict__ part)
{
    __shared__ float lds[(2 * V + 1) * kThreads];
    const Place at = place(d);
    const long long items = d.N * d.chunks;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long n = item / d.chunks, chunk = item - n * d.chunks, first = chunk * d.chunk, end = min(first + d.chunk, d.P);
        const TX* base = x + (size_t)(n * d.P) * d.xs + at.slot * V;
        const float* occ = MASK ? d.occ + n * d.P : nullptr;
        Sums<V> sums;
        if (at.in) {
            Pack<TX, V> v[kUnroll<V>];
            bool on[kUnroll<V>];
            sweep<kUnroll<V>>(d, first, end, at.row,
                  [&](int u, long long p, bool in) {
                      on[u] = in && (!MASK || occ[p] > 0.0f);
                      if (on[u]) load<TX, V>(base + p * d.xs, v[u]);
                  },
                  [&](int u, long long, bool) {
                      if (on[u]) sums.add(v[u]);
                  });
        }
        float count = sums.count, mean[V], m2[V];
        sums.close(mean, m2);
        join_rows<V, kThreads>(d, at, count, mean, m2, lds);
        if (at.in && at.row == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) part[(size_t)(n * d.C + at.slot * V + j) * d.chunks + chunk] = f32x4{count, mean[j], m2[j], 0.0f};
        }
    }
}

constexpr int kJoinThreads = 512;
__device__ __forceinline__ double block_sum(double v, double* lds)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kJoinThreads / 64; ++k) sum += lds[k];
    return sum;
}

// Joins a group's parts: one workgroup a (sample, group) -> stats[(n G + g) 2] = mean, rstd.
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(NormDev d, const f32x4* __restrict__ part, float* __restrict__ stats)
{
    __shared__ double lds[kJoinThreads / 64];
    const long long groups = d.N * d.G;
    for (long long k = blockIdx.x; k < groups; k += gridDim.x) {
        // (the parts of a group lie one behind the other)
        const f32x4* from = part + (size_t)k * d.Cg * d.chunks;
        double cnt = 0.0, sum = 0.0, sq = 0.0;
        const long long all = (long long)d.chunks * d.Cg;
        for (long long i = threadIdx.x; i < all; i += 4 * kJoinThreads) {   // (four parts are asked for at a time)
            f32x4 p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) p[u] = i + u * kJoinThreads < all ? from[i + u * kJoinThreads] : f32x4{};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const double c = p[u][0], m = p[u][1];
                cnt += c;
                sum += c * m;
                sq += (double)p[u][2] + c * m * m;
            }
        }
        cnt = block_sum(cnt, lds);
        sum = block_sum(sum, lds);
        sq = block_sum(sq, lds);
        if (threadIdx.x == 0) {
            float mean, rstd;
            statistics_of(cnt, sum, sq, d.eps, mean, rstd);
            stats[2 * k] = mean;
            stats[2 * k + 1] = rstd;
        }
    }
}

// Pass 2 of the forward.
template <class TX, class TY, int V, bool MASK>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormDev d, const TX* x, TY* y, const float* __restrict__ stats)
{
    const Place at = place(d);
    if (!at.in) return;
    Slot<V> slot;
    slot.parameters(d, at.slot);
    const long long items = d.N * d.chunks;
    for (long long k = blockIdx.x; k < items; k += gridDim.x) {
        const long long item = items - 1 - k, n = item / d.chunks, first = (item - n * d.chunks) * d.chunk, end = min(first + d.chunk, d.P);
        const TX* base = x + (size_t)(n * d.P) * d.xs + at.slot * V;
        TY* out = y + (size_t)(n * d.P) * d.ys + at.slot * V;
        const float* occ = MASK ? d.occ + n * d.P : nullptr;
        slot.statistics(d, at.slot, stats + n * d.G * 2);
        float scale[V];
#pragma unroll
        for (int j = 0; j < V; ++j) scale[j] = slot.rstd[j] * slot.gamma[j];
        with_act(d.act, [&](auto act) {
            Pack<TX, V> v[kUnroll<V>];   // (as they are stored: converted where they are used)
            bool on[kUnroll<V>];
            sweep<kUnroll<V>>(d, first, end, at.row,
                  [&](int u, long long p, bool in) {
                      on[u] = in && (!MASK || occ[p] > 0.0f);
                      if (on[u]) load<TX, V>(base + p * d.xs, v[u]);
                  },
                  [&](int u, long long p, bool in) {
                      if (!in) return;
                      float r[V];
#pragma unroll
                      for (int j = 0; j < V; ++j)
                          r[j] = on[u] ? activate<decltype(act)::value>(fmaf(to_f32(v[u].v[j]) - slot.mean[j], scale[j], slot.beta[j])) : 0.0f;
                      store<TY, V>(out + p * d.ys, r);
                  });
        });
    }
}

// Pass 1 of the backward: (sum g, sum g xh) of every channel of every item -> part[((n C + c) chunks + chunk) 2], and the item's count.
template <class TX, class TY, int V, bool MASK>
__global__ __launch_bounds__(kThreads) void norm_grad_sums_kernel(NormDev d, const TX* __restrict__ x, const TY* __restrict__ dy,
                                                                  const float* __restrict__ stats, f32x2* __restrict__ part,
                                                                  float* __restrict__ counts)
{
    __shared__ float lds[(2 * V + 1) * kThreads];
    const Place at = place(d);
    Slot<V> slot;
    if (at.in) slot.parameters(d, at.slot);
    const long long items = d.N * d.chunks;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long n = item / d.chunks, chunk = item - n * d.chunks, first = chunk * d.chunk, end = min(first + d.chunk, d.P);
        float sg[V], sx[V], count = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) sg[j] = sx[j] = 0.0f;
        if (at.in) {
            const TX* base = x + (size_t)(n * d.P) * d.xs + at.slot * V;
            const TY* up = dy + (size_t)(n * d.P) * d.ys + at.slot * V;
            const float* occ = MASK ? d.occ + n * d.P : nullptr;
            slot.statistics(d, at.slot, stats + n * d.G * 2);
            with_act(d.act, [&](auto act) {
                Pack<TX, V> v[kUnroll<V>];   // (as they are stored: converted where they are used)
                Pack<TY, V> w[kUnroll<V>];
                bool on[kUnroll<V>];
                sweep<kUnroll<V>>(d, first, end, at.row,
                      [&](int u, long long p, bool in) {
                          on[u] = in && (!MASK || occ[p] > 0.0f);
                          if (on[u]) {
                              load<TX, V>(base + p * d.xs, v[u]);
                              load<TY, V>(up + p * d.ys, w[u]);
                          }
                      },
                      [&](int u, long long, bool) {
                          if (!on[u]) return;
#pragma unroll
                          for (int j = 0; j < V; ++j) {
                              const float xh = (to_f32(v[u].v[j]) - slot.mean[j]) * slot.rstd[j];
                              const float g = to_f32(w[u].v[j]) * slope<decltype(act)::value>(fmaf(xh, slot.gamma[j], slot.beta[j]));
                              sg[j] += g;
                              sx[j] = fmaf(g, xh, sx[j]);
                          }
                          count += 1.0f;
                      });
            });
        }
        add_rows<V, kThreads>(d, at, count, sg, sx, lds);
        if (at.in && at.row == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) part[(size_t)(n * d.C + at.slot * V + j) * d.chunks + chunk] = f32x2{sg[j], sx[j]};
            if (at.slot == 0) counts[item] = count;
        }
    }
}

// Joins the backward's parts: one workgroup a (sample, group), a wave a channel at a time.  chan[(n C + c) 2] = sums of a
// channel, means[(n G + g) 2] = S1 / count, S2 / count; with a single sample the parameters' gradients are added here.
__global__ __launch_bounds__(kJoinThreads) void norm_grad_join_kernel(NormDev d, const f32x2* __restrict__ part, const float* __restrict__ counts,
                                                                      double* __restrict__ chan, float* __restrict__ means, float* d_gamma,
                                                                      float* d_beta)
{
    __shared__ double lds[kJoinThreads / 64];
    const long long groups = d.N * d.G;
    for (long long k = blockIdx.x; k < groups; k += gridDim.x) {
        const long long n = k / d.G;
        const int g = (int)(k - n * d.G);
        double cnt = 0.0;
        for (int i = threadIdx.x; i < d.chunks; i += kJoinThreads) cnt += (double)counts[n * d.chunks + i];
        double s1 = 0.0, s2 = 0.0;
        for (int j = threadIdx.x >> 6; j < d.Cg; j += kJoinThreads / 64) {
            const int c = g * d.Cg + j;
            const f32x2* from = part + (size_t)(n * d.C + c) * d.chunks;
            double a = 0.0, b = 0.0;
            for (int i = threadIdx.x & 63; i < d.chunks; i += 8 * 64) {   // (eight parts are asked for at a time)
                f32x2 p[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) p[u] = i + 64 * u < d.chunks ? from[i + 64 * u] : f32x2{};
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    a += (double)p[u][0];
                    b += (double)p[u][1];
                }
            }
            a = wave_sum(a);
            b = wave_sum(b);
            if ((threadIdx.x & 63) == 0) {
                const double gamma = d.gamma ? (double)d.gamma[c] : 1.0;
                s1 += gamma * a;
                s2 += gamma * b;
                if (d.N > 1) {
                    chan[(n * d.C + c) * 2] = a;
                    chan[(n * d.C + c) * 2 + 1] = b;
                } else {
                    if (d_beta) d_beta[c] = (float)((double)d_beta[c] + a);
                    if (d_gamma) d_gamma[c] = (float)((double)d_gamma[c] + b);
                }
            }
        }
        cnt = block_sum(cnt, lds) * d.Cg;
        s1 = block_sum(s1, lds);
        s2 = block_sum(s2, lds);
        if (threadIdx.x == 0) {
            means[2 * k] = cnt > 0.0 ? (float)(s1 / cnt) : 0.0f;
            means[2 * k + 1] = cnt > 0.0 ? (float)(s2 / cnt) : 0.0f;
        }
    }
}

// Gradients of the parameters over several samples, whose sums are added in order (four samples are asked for at a time).
__device__ __forceinline__ void add_parameters(const NormDev& d, const double* __restrict__ chan, float* d_gamma, float* d_beta)
{
    for (int c = threadIdx.x; c < d.C; c += kThreads) {
        double a = 0.0, b = 0.0;
        for (long long n = 0; n < d.N; n += 4) {
            double v[4][2];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int k = 0; k < 2; ++k) v[u][k] = n + u < d.N ? chan[((n + u) * d.C + c) * 2 + k] : 0.0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                a += v[u][0];
                b += v[u][1];
            }
        }
        if (d_beta) d_beta[c] = (float)((double)d_beta[c] + a);
        if (d_gamma) d_gamma[c] = (float)((double)d_gamma[c] + b);
    }
}
__global__ __launch_bounds__(kThreads) void norm_params_kernel(NormDev d, const double* __restrict__ chan, float* d_gamma, float* d_beta)
{
    add_parameters(d, chan, d_gamma, d_beta);
}

// Pass 2 of the backward.  `chan` not NULL: the first workgroup adds up the parameters' gradients.
template <class TX, class TY, int V, bool MASK>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormDev d, const TX* x, const TY* dy, TX* dx,
                                                             const float* __restrict__ stats, const float* __restrict__ means,
                                                             const double* __restrict__ chan, float* d_gamma, float* d_beta)
{
    if (chan && blockIdx.x == 0 && blockIdx.y == 0) add_parameters(d, chan, d_gamma, d_beta);
    const Place at = place(d);
    if (!at.in) return;
    Slot<V> slot;
    slot.parameters(d, at.slot);
    const long long items = d.N * d.chunks;
    for (long long k = blockIdx.x; k < items; k += gridDim.x) {
        const long long item = items - 1 - k, n = item / d.chunks, first = (item - n * d.chunks) * d.chunk, end = min(first + d.chunk, d.P);
        const TX* base = x + (size_t)(n * d.P) * d.xs + at.slot * V;
        const TY* up = dy + (size_t)(n * d.P) * d.ys + at.slot * V;
        TX* out = dx + (size_t)(n * d.P) * d.xs + at.slot * V;
        const float* occ = MASK ? d.occ + n * d.P : nullptr;
        slot.statistics(d, at.slot, stats + n * d.G * 2);
        // d_x = rstd (gamma g - m1 - xh m2)
        float scale[V], m1[V], m2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const long long g = n * d.G + (at.slot * V + j) / d.Cg;
            scale[j] = slot.rstd[j] * slot.gamma[j];
            m1[j] = slot.rstd[j] * means[2 * g];
            m2[j] = slot.rstd[j] * means[2 * g + 1];
        }
        with_act(d.act, [&](auto act) {
            Pack<TX, V> v[kUnroll<V>];   // (as they are stored: converted where they are used)
            Pack<TY, V> w[kUnroll<V>];
            bool on[kUnroll<V>];
            sweep<kUnroll<V>>(d, first, end, at.row,
                  [&](int u, long long p, bool in) {
                      on[u] = in && (!MASK || occ[p] > 0.0f);
                      if (on[u]) {
                          load<TX, V>(base + p * d.xs, v[u]);
                          load<TY, V>(up + p * d.ys, w[u]);
                      }
                  },
                  [&](int u, long long p, bool in) {
                      if (!in) return;
                      float r[V];
#pragma unroll
                      for (int j = 0; j < V; ++j) {
                          const float xh = (to_f32(v[u].v[j]) - slot.mean[j]) * slot.rstd[j];
                          const float g = to_f32(w[u].v[j]) * slope<decltype(act)::value>(fmaf(xh, slot.gamma[j], slot.beta[j]));
                          r[j] = on[u] ? fmaf(scale[j], g, -fmaf(xh, m2[j], m1[j])) : 0.0f;
                      }
                      store<TX, V>(out + p * d.xs, r);
                  });
        });
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int dtype_bytes(int t) { return t == LP_F32 ? 4 : 2; }

lp_status validate(const lp_group_norm* q, NormDev* d)
{
    if (!q) return fail(LP_ERR_INVALID_ARG, "norm must not be NULL");
    if (q->N < 0 || q->P < 0) return fail(LP_ERR_INVALID_ARG, "norm->N and norm->P must be >= 0");
    if (q->C < 1 || q->G < 1 || q->C % q->G) return fail(LP_ERR_INVALID_ARG, "norm->G must be >= 1 and divide norm->C");
    if (q->act < LP_ACT_NONE || q->act > LP_ACT_GELU) return fail(LP_ERR_INVALID_ARG, "norm->act must be an lp_act");
    if (!std::isfinite(q->eps) || q->eps < 0.0f) return fail(LP_ERR_INVALID_ARG, "norm->eps must be finite and >= 0");
    for (int t : {q->x_dtype, q->y_dtype})
        if (t != LP_F32 && t != LP_BF16 && t != LP_F16)
            return fail(LP_ERR_INVALID_ARG, "norm->x_dtype and norm->y_dtype must be LP_F32, LP_BF16 or LP_F16");
    if (q->x_dtype != q->y_dtype && q->x_dtype != LP_F32)
        return fail(LP_ERR_UNSUPPORTED, "norm->y_dtype must be norm->x_dtype unless that is LP_F32");
    const long long xs = q->x_stride ? q->x_stride : q->C, ys = q->y_stride ? q->y_stride : q->C;
    if (xs < q->C || ys < q->C) return fail(LP_ERR_INVALID_ARG, "norm->x_stride and norm->y_stride must be 0 or >= norm->C");
    // offsets in bytes are kept in 64 bits
    const double most = (double)q->N * (double)q->P * (double)(xs > ys ? xs : ys) * 4.0;
    if (most > 4e18 || (double)q->N * (double)q->C > 1e12) return fail(LP_ERR_UNSUPPORTED, "norm: tensors beyond 64-bit offsets");
    std::memset(d, 0, sizeof(*d));
    d->N = q->N; d->P = q->P; d->C = q->C; d->G = q->G; d->Cg = q->C / q->G;
    d->xs = xs; d->ys = ys; d->gamma = q->gamma; d->beta = q->beta; d->occ = q->occupancy; d->eps = q->eps; d->act = q->act;
    return LP_OK;
}

// Divides the work for slots of V channels.  The number of items does not depend on V by more than rounding: `most` is what
// the workspace has room for.
void divide(NormDev* d, int V, int n_cu)
{
    d->slots = d->C / V;
    d->zblocks = (d->slots + kThreads - 1) / kThreads;
    d->rows = d->zblocks > 1 ? 1 : kThreads / d->slots;
    // eight workgroups a compute unit keep enough loads in flight; no fewer than eight positions a thread, at most 2^22 an item
    // (counts are exact in fp32)
    const long long target = ((long long)8 * n_cu + d->N - 1) / (d->N > 0 ? d->N : 1);
    long long most = (d->P + 8ll * d->rows - 1) / (8ll * d->rows);
    long long chunks = target < most ? target : most;
    const long long least = (d->P + (1ll << 22) - 1) >> 22;
    if (chunks < least) chunks = least;
    if (chunks < 1) chunks = 1;
    d->chunk = (d->P + chunks - 1) / chunks;
    d->chunk = (d->chunk + d->rows - 1) / d->rows * d->rows;
    if (d->chunk < 1) d->chunk = 1;
    d->chunks = (int)((d->P + d->chunk - 1) / d->chunk);
    if (d->chunks < 1) d->chunks = 1;
}

long long most_items(const NormDev& d, int n_cu)
{
    long long most = 0;
    for (int V = 1; V <= 8; V *= 2) {
        if (d.C % V) break;
        NormDev t = d;
        divide(&t, V, n_cu);
        if (t.N * t.chunks > most) most = t.N * t.chunks;
    }
    return most;
}

// Whether a sample fits the registers of a workgroup: then `d` is divided for that.  They hold 32 Ki values in slots of four channels (fp32,
// or 16 bits that are aligned to eight bytes only), 16 Ki in slots of eight or one, less where C / V does not divide 1024.
// A plane of 32 x 32 x 16 in fp32 takes 9 us like that and 16 us in three launches.
bool hold(NormDev* d, int V)
{
    const int held = V == 8 ? 2 : V == 4 ? 8 : 16;
    if (d->C / V > kSmallThreads || d->C > kSmallThreads || d->N > kMaxGrid) return false;
    const int rows = kSmallThreads / (d->C / V);
    if (d->P > (long long)rows * held) return false;
    d->slots = d->C / V;
    d->zblocks = 1;
    d->rows = rows;
    return true;
}

struct Sizes {
    size_t part, counts, chan, means, stats, fwd, bwd;
};
Sizes sizes(const NormDev& d, int n_cu)
{
    Sizes s;
    const size_t items = (size_t)most_items(d, n_cu);
    s.part = align256(items * d.C * sizeof(f32x4));
    s.counts = align256(items * sizeof(float));
    s.chan = align256((size_t)d.N * d.C * 2 * sizeof(double));
    s.means = s.stats = align256((size_t)d.N * d.G * 2 * sizeof(float));
    s.fwd = s.part + s.stats;
    s.bwd = s.part + s.counts + s.chan + s.means;
    // samples held in registers whatever the slots need no parts, and a single one nothing at all
    bool small = true;
    for (int V = 1; V <= 8; V *= 2) {
        NormDev t = d;
        if (d.C % V == 0 && V != 2 && !hold(&t, V)) small = false;
    }
    if (small) {
        s.part = s.counts = s.means = s.stats = s.fwd = 0;
        if (d.N == 1) s.chan = 0;
        s.bwd = s.chan;
    }
    return s;
}

// The widest slot that channels, strides and addresses allow: 16 bytes of x.
int slot_width(const NormDev& d, int x_bytes, int y_bytes, std::initializer_list<const void*> xs, std::initializer_list<const void*> ys)
{
    for (int V = 16 / x_bytes; V > 1; V = V == 8 ? 4 : 1) {
        bool ok = d.C % V == 0 && d.xs % V == 0 && d.ys % V == 0;
        for (const void* p : xs) ok = ok && (uintptr_t)p % (V * x_bytes) == 0;
        for (const void* p : ys) ok = ok && (uintptr_t)p % (V * y_bytes) == 0;
        if (ok) return V;
    }
    return 1;
}

// Calls f with the types, the slot width and whether there is an occupancy as constants.
template <class T> struct Type { using type = T; };
template <class F, class X, class Y, int... Vs>
void with_width(int V, bool mask, F&& f, Type<X> x, Type<Y> y, std::integer_sequence<int, Vs...>)
{
    auto one = [&](auto v) {
        if (v.value != V) return;
        if (mask) f(x, y, v, std::true_type()); else f(x, y, v, std::false_type());
    };
    (one(std::integral_constant<int, Vs>()), ...);
}
template <class F>
void dispatch(int x_dtype, int y_dtype, int V, bool mask, F&& f)
{
    using W4 = std::integer_sequence<int, 1, 4>;
    using W8 = std::integer_sequence<int, 1, 4, 8>;
    if (x_dtype == LP_BF16) with_width(V, mask, f, Type<__bf16>(), Type<__bf16>(), W8());
    else if (x_dtype == LP_F16) with_width(V, mask, f, Type<_Float16>(), Type<_Float16>(), W8());
    else if (y_dtype == LP_BF16) with_width(V, mask, f, Type<float>(), Type<__bf16>(), W4());
    else if (y_dtype == LP_F16) with_width(V, mask, f, Type<float>(), Type<_Float16>(), W4());
    else with_width(V, mask, f, Type<float>(), Type<float>(), W4());
}

unsigned grid_of(long long items) { return (unsigned)(items < kMaxGrid ? items : kMaxGrid); }

lp_status launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LP_OK : fail(LP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

lp_status forward(const lp_group_norm* q, const void* x, void* y, float* stats, void* workspace, size_t workspace_bytes, hipStream_t s)
{
    NormDev d;
    lp_status st = validate(q, &d);
    if (st != LP_OK) return st;
    if (d.N == 0 || d.P == 0) return LP_OK;
    if (!x || !y) return fail(LP_ERR_INVALID_ARG, "x and y must not be NULL");
    std::string err;
    int n_cu = 0;
    if (compute_units(&n_cu, &err)) return fail(LP_ERR_HIP, err);
    const Sizes size = sizes(d, n_cu);
    if (size.fwd && (!workspace || workspace_bytes < size.fwd))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_group_norm_workspace_bytes");
    if (size.fwd && (uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const int V = slot_width(d, dtype_bytes(q->x_dtype), dtype_bytes(q->y_dtype), {x}, {y});
    const bool small = hold(&d, V);
    if (!small) divide(&d, V, n_cu);
    f32x4* part = (f32x4*)workspace;
    float* used = stats ? stats : (float*)((char*)workspace + size.part);
    const dim3 grid(grid_of(d.N * d.chunks), d.zblocks);
    dispatch(q->x_dtype, q->y_dtype, V, d.occ != nullptr, [&](auto tx, auto ty, auto v, auto mask) {
        using TX = typename decltype(tx)::type;
        using TY = typename decltype(ty)::type;
        constexpr int W = decltype(v)::value;
        constexpr bool M = decltype(mask)::value;
        if (small) {
            hipLaunchKernelGGL((norm_small_kernel<TX, TY, W, M>), dim3((unsigned)d.N), dim3(kSmallThreads), 0, s, d, (const TX*)x, (TY*)y, stats);
            return;
        }
        hipLaunchKernelGGL((norm_stats_kernel<TX, W, M>), grid, dim3(kThreads), 0, s, d, (const TX*)x, part);
        hipLaunchKernelGGL(norm_join_kernel, dim3(grid_of(d.N * d.G)), dim3(kJoinThreads), 0, s, d, part, used);
        hipLaunchKernelGGL((norm_apply_kernel<TX, TY, W, M>), grid, dim3(kThreads), 0, s, d, (const TX*)x, (TY*)y, used);
    });
    return launched("group norm forward launch");
}

lp_status backward(const lp_group_norm* q, const void* x, const float* stats, const void* dy, void* dx, float* d_gamma, float* d_beta,
                   void* workspace, size_t workspace_bytes, hipStream_t s)
{
    NormDev d;
    lp_status st = validate(q, &d);
    if (st != LP_OK) return st;
    if (d.N == 0 || d.P == 0) return LP_OK;
    if (!x || !stats || !dy) return fail(LP_ERR_INVALID_ARG, "x, stats and d_y must not be NULL");
    std::string err;
    int n_cu = 0;
    if (compute_units(&n_cu, &err)) return fail(LP_ERR_HIP, err);
    const Sizes size = sizes(d, n_cu);
    if (size.bwd && (!workspace || workspace_bytes < size.bwd))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_group_norm_workspace_bytes");
    if (size.bwd && (uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const int V = slot_width(d, dtype_bytes(q->x_dtype), dtype_bytes(q->y_dtype), {x, dx}, {dy});
    const bool small = hold(&d, V);
    if (!small) divide(&d, V, n_cu);
    char* at = (char*)workspace;
    f32x2* part = (f32x2*)at;
    float* counts = (float*)(at += size.part);
    double* chan = (double*)(at += size.counts);
    float* means = (float*)(at += size.chan);
    const dim3 grid(grid_of(d.N * d.chunks), d.zblocks);
    dispatch(q->x_dtype, q->y_dtype, V, d.occ != nullptr, [&](auto tx, auto ty, auto v, auto mask) {
        using TX = typename decltype(tx)::type;
        using TY = typename decltype(ty)::type;
        constexpr int W = decltype(v)::value;
        constexpr bool M = decltype(mask)::value;
        const bool params = (d_gamma || d_beta) && d.N > 1;
        if (small) {
            hipLaunchKernelGGL((norm_small_grad_kernel<TX, TY, W, M>), dim3((unsigned)d.N), dim3(kSmallThreads), 0, s, d, (const TX*)x,
                               (const TY*)dy, (TX*)dx, stats, chan, d_gamma, d_beta);
        } else {
            hipLaunchKernelGGL((norm_grad_sums_kernel<TX, TY, W, M>), grid, dim3(kThreads), 0, s, d, (const TX*)x, (const TY*)dy, stats,
                               part, counts);
            hipLaunchKernelGGL(norm_grad_join_kernel, dim3(grid_of(d.N * d.G)), dim3(kJoinThreads), 0, s, d, part, counts, chan, means,
                               d_gamma, d_beta);
        }
        if (params && (small || !dx))
            hipLaunchKernelGGL(norm_params_kernel, dim3(1), dim3(kThreads), 0, s, d, chan, d_gamma, d_beta);
        if (small) return;
        if (dx)
            hipLaunchKernelGGL((norm_grad_kernel<TX, TY, W, M>), grid, dim3(kThreads), 0, s, d, (const TX*)x, (const TY*)dy, (TX*)dx,
                               stats, means, params ? chan : nullptr, d_gamma, d_beta);
    });
    return launched("group norm backward launch");
}

}  // namespace

}  // namespace lp

extern "C" {

lp_status lp_group_norm_workspace_bytes(const lp_group_norm* norm, size_t* fwd_bytes, size_t* bwd_bytes)
try {
    lp::NormDev d;
    const lp_status st = lp::validate(norm, &d);
    if (st != LP_OK) return st;
    std::string err;
    int n_cu = 0;
    if (lp::compute_units(&n_cu, &err)) return lp::fail(LP_ERR_HIP, err);
    const lp::Sizes size = lp::sizes(d, n_cu);
    if (fwd_bytes) *fwd_bytes = size.fwd;
    if (bwd_bytes) *bwd_bytes = size.bwd;
    return LP_OK;
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_group_norm_fwd(const lp_group_norm* norm, const void* x, void* y, float* stats, void* workspace, size_t workspace_bytes,
                            void* stream)
try {
    return lp::forward(norm, x, y, stats, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_group_norm_bwd(const lp_group_norm* norm, const void* x, const float* stats, const void* d_y, void* d_x, float* d_gamma,
                            float* d_beta, void* workspace, size_t workspace_bytes, void* stream)
try {
    return lp::backward(norm, x, stats, d_y, d_x, d_gamma, d_beta, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

}  // extern "C"
