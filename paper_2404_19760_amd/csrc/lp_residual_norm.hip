// The norms around a residual block, with its gate and the residual sum, forward and backward.
//
//     u = post_gamma fh, fh = norm(f)   (or u = fh = f),   s = alpha h + gate u,   xh = norm(s),   y = gamma xh + beta
//
// and with e = gamma d_y, means over a position's channels,
//     g = d_s + rstd (e - xh mean(e xh) [- mean(e)]),   d_h = alpha g,   d_u = gate g,
//     d_f = rstd_f (k - fh mean(k fh) [- mean(k)]), k = post_gamma d_u   (or d_f = d_u),
//     d_gamma = sum d_y xh,   d_beta = sum d_y,   T = sum g fh:  d_gate = post_gamma T,   d_post_gamma = gate T
// ([..]: of a layer norm).  The gate's and the post norm's gradients come from the same sums T, a sample at a time.
//
// What bounds it: memory.  A position stays in the registers of a group of lanes (of a wave, or of a workgroup beyond 512 channels),
// so every tensor is read or written once; the backward computes s and both norms again from h and f, which costs some
// sums over lanes and spares two numbers a position from being kept.  Lanes hold slots of V neighbouring channels (16 bytes of h where channels and alignment
// allow).  A workgroup takes the positions of a part of a sample; column sums stay in the lanes' registers meanwhile, are
// joined over the workgroup's groups at the end and over the workgroups, in fp64, by a second kernel, in a fixed order.
//
// Measured: gradients of 65536 x 512 in bf16 with both norms 83 us for 0.40 GB (4.9 TB/s), of 24 x 256^2 x 32, sums in fp32 and blocks in bf16, 184 us for
// 0.91 GB; forward of 131979 x 72 in fp16 18 us for 76 MB.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "lp_kernels.h"
#include "lp_lanes.h"

namespace lp {

namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 8;           // channels of a position that a lane holds; beyond kWideThreads of them 2 kHeld
constexpr int kWaveChannels = 64 * kHeld, kWideThreads = 512;
constexpr int kJoinThreads = 1024;
constexpr unsigned kMaxGrid = 1u << 20;
// Where a call moves more than the Infinity Cache holds, results are stored past the caches: they would only drive out what is yet to
// be read (gradients of 65536 x 512 in bf16, 0.4 GB: 101 -> 90 us).
constexpr double kCacheBytes = 256e6;

struct NormDev {
    long long N, P;                // samples, positions of a sample (a gate that is the same for all: one sample)
    int C, layer, post;
    int lanes, groups;             // lanes of a position (power of two; all threads beyond kWaveChannels), positions a workgroup takes at a time
    float eps, alpha;
    long long hs, fs, ys;
    const float *post_gamma, *gate, *gamma, *beta;
    long long chunk;               // positions of an item
    int chunks;                    // items of a sample
    int past_cache;                // results are stored past the caches
};

template <class T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

// A group of lanes and where a lane stands in it.
template <bool WIDE>
struct Group {
    int lanes, lane, index;
    float* lds;
    __device__ __forceinline__ Group(const NormDev& d, float* lds) : lanes(d.lanes), lds(lds)
    {
        if (WIDE) {
            lane = threadIdx.x;
            index = 0;
        } else {
            lane = threadIdx.x & (lanes - 1);
            index = threadIdx.x / lanes;
        }
    }
    // Sums over the group's lanes, K at once; every lane gets them.
    template <int K>
    __device__ __forceinline__ void sum(float (&v)[K]) const
    {
        lane_sums(v, WIDE ? 64 : lanes);
        if (!WIDE) return;
        const int waves = blockDim.x >> 6;
        __syncthreads();   // (the sums before have been read)
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * 16 + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.0f;
            for (int w = 0; w < waves; ++w) v[k] += lds[k * 16 + w];
        }
    }
};

// A lane's slots: slot r holds channels ((r lanes + lane) V) ..  WHOLE: C is a multiple of V; else the last slot's values are moved one by
// one.  Slots need not be aligned to their size.
template <bool WHOLE, class T, int V, int R, class G>
__device__ __forceinline__ void load(const NormDev& d, const G& g, const T* row, Pack<T, V> (&out)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * g.lanes + g.lane) * V;
        if (c + (WHOLE ? 0 : V - 1) < d.C) {
            __builtin_memcpy(&out[r], row + c, sizeof(out[r]));
        } else if (!WHOLE) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < d.C) out[r].v[j] = row[c + j];
        }
    }
}
template <bool WHOLE, class T, int V, int R, class G>
__device__ __forceinline__ void store(const NormDev& d, const G& g, T* row, const float (&v)[R * V])
{
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * g.lanes + g.lane) * V;
        Pack<T, V> q;
#pragma unroll
        for (int j = 0; j < V; ++j) q.v[j] = (T)v[r * V + j];   // rounded once
        if (c + (WHOLE ? 0 : V - 1) < d.C) {
            if (d.past_cache) {
                typedef uint32_t Any __attribute__((ext_vector_type(sizeof(T) * V / 4), aligned(2)));
                asm volatile("" ::: "memory");   // (with nothing around it both stores would become one ordinary one)
                __builtin_nontemporal_store(__builtin_bit_cast(Any, q), (Any*)(row + c));
                asm volatile("" ::: "memory");
            } else {
                __builtin_memcpy(row + c, &q, sizeof(q));
            }
        } else if (!WHOLE) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < d.C) row[c + j] = q.v[j];
        }
    }
}
// Whether a lane's value is one of a channel.
template <bool WHOLE, int V, class G>
__device__ __forceinline__ bool on(const NormDev& d, const G& g, int r, int j) { return (r * g.lanes + g.lane) * V + (WHOLE ? 0 : j) < d.C; }

// A parameter's values (NULL: `none`); lanes without channels hold zeros.
template <bool WHOLE, int V, int R, class G>
__device__ __forceinline__ void parameter(const NormDev& d, const G& g, const float* p, float none, float (&out)[R * V])
{
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * g.lanes + g.lane) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) out[r * V + j] = on<WHOLE, V>(d, g, r, j) ? (p ? p[c + j] : none) : 0.0f;
    }
}
template <bool WHOLE, class T, int V, int R, class G>
__device__ __forceinline__ void widen(const NormDev& d, const G& g, const Pack<T, V> (&in)[R], float (&out)[R * V])
{
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < V; ++j) out[r * V + j] = on<WHOLE, V>(d, g, r, j) ? (float)in[r].v[j] : 0.0f;   // (zeros behind the last channel: they add nothing to sums)
}

// v becomes norm(v); the result is what it was multiplied with.  Variances are of differences to the mean.
template <bool WHOLE, int V, int R, class G>
__device__ __forceinline__ float normalise(const NormDev& d, const G& g, float (&v)[R * V])
{
    const float over = 1.0f / (float)d.C;
    if (d.layer) {
        float sum[1] = {0.0f};
#pragma unroll
        for (int e = 0; e < R * V; ++e) sum[0] += v[e];
        g.sum(sum);
        const float mean = sum[0] * over;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < V; ++j) v[r * V + j] = on<WHOLE, V>(d, g, r, j) ? v[r * V + j] - mean : 0.0f;
    }
    float squares[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < R * V; ++e) squares[0] = fmaf(v[e], v[e], squares[0]);
    g.sum(squares);
    const float rstd = 1.0f / sqrtf(fmaf(squares[0], over, d.eps));
#pragma unroll
    for (int e = 0; e < R * V; ++e) v[e] *= rstd;
    return rstd;
}

// The gradient of norm's argument for that of its result, in place.
template <int V, int R, class G>
__device__ __forceinline__ void normalise_grad(const NormDev& d, const G& g, const float (&xh)[R * V], float rstd, float (&e)[R * V])
{
    const float over = 1.0f / (float)d.C;
    float sums[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < R * V; ++k) {
        sums[0] = fmaf(e[k], xh[k], sums[0]);
        sums[1] += e[k];
    }
    g.sum(sums);
    const float along = sums[0] * over, mean = d.layer ? sums[1] * over : 0.0f;
#pragma unroll
    for (int k = 0; k < R * V; ++k) e[k] = rstd * (e[k] - fmaf(xh[k], along, mean));
}

template <class TH, class TF, int V, int R, bool WIDE, bool WHOLE>
__global__ __launch_bounds__(WIDE ? kWideThreads : kThreads) void residual_norm_kernel(NormDev d, const TH* h, const TF* f, TH* s, TF* y)
{
    constexpr int kAhead = WIDE || R > 1 ? 1 : 2;
    __shared__ float lds[2 * 16];
    const Group<WIDE> g(d, lds);
    float post_gamma[R * V], gate[R * V], gamma[R * V], beta[R * V];
    parameter<WHOLE, V, R>(d, g, d.post_gamma, 1.0f, post_gamma);
    parameter<WHOLE, V, R>(d, g, d.gamma, 1.0f, gamma);
    parameter<WHOLE, V, R>(d, g, d.beta, 0.0f, beta);
    const long long items = d.N * d.chunks;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long n = item / d.chunks, first = (item - n * d.chunks) * d.chunk, end = min(d.P, first + d.chunk);
        parameter<WHOLE, V, R>(d, g, d.gate ? d.gate + n * d.C : nullptr, 1.0f, gate);
        // (the next positions are asked for before this one's sums)
        Pack<TH, V> hp[R], h_next[kAhead][R];
        Pack<TF, V> fp[R], f_next[kAhead][R];
        const long long start = n * d.P + first + g.index;
        const TH* h_at = h + start * d.hs;
        const TF* f_at = f + start * d.fs;
        TH* s_at = s + start * d.hs;
        TF* y_at = y + start * d.ys;
        auto ask = [&](long long p, Pack<TH, V> (&hn)[R], Pack<TF, V> (&fn)[R]) {
            if (p < end) {
                load<WHOLE, TH, V, R>(d, g, h_at, hn);
                if (f) load<WHOLE, TF, V, R>(d, g, f_at, fn);
            }
            h_at += d.groups * d.hs;
            f_at += d.groups * d.fs;
        };
        const long long mine = first + g.index;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ask(mine + u * d.groups, h_next[u], f_next[u]);
        for (long long p = mine; p < end; p += d.groups) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                hp[r] = h_next[0][r];
                fp[r] = f_next[0][r];
#pragma unroll
                for (int u = 1; u < kAhead; ++u) {
                    h_next[u - 1][r] = h_next[u][r];
                    f_next[u - 1][r] = f_next[u][r];
                }
            }
            ask(p + kAhead * d.groups, h_next[kAhead - 1], f_next[kAhead - 1]);
            float v[R * V], t[R * V];
            if (f) {
                widen<WHOLE, TF, V, R>(d, g, fp, v);
                if (d.post) {
                    normalise<WHOLE, V, R>(d, g, v);
#pragma unroll
                    for (int e = 0; e < R * V; ++e) v[e] *= post_gamma[e];
                }
                widen<WHOLE, TH, V, R>(d, g, hp, t);
#pragma unroll
                for (int e = 0; e < R * V; ++e) t[e] = fmaf(gate[e], v[e], d.alpha * t[e]);
            } else {
                widen<WHOLE, TH, V, R>(d, g, hp, t);
#pragma unroll
                for (int e = 0; e < R * V; ++e) t[e] *= d.alpha;
            }
            if (s) store<WHOLE, TH, V, R>(d, g, s_at, t);
            s_at += d.groups * d.hs;
            if (!y) continue;
            normalise<WHOLE, V, R>(d, g, t);
#pragma unroll
            for (int e = 0; e < R * V; ++e) t[e] = fmaf(gamma[e], t[e], beta[e]);
            store<WHOLE, TF, V, R>(d, g, y_at, t);
            y_at += d.groups * d.ys;
        }
    }
}

// Column sums of an item: [3][C] of d_y xh, d_y and g fh.
template <class TH, class TF, int V, int R, bool WIDE, bool WHOLE>
__global__ __launch_bounds__(WIDE ? kWideThreads : kThreads, R * V <= kHeld ? 3 : 2) void residual_norm_grad_kernel(NormDev d, const TH* h, const TF* f, const TH* d_s,
                                                                                   const TF* d_y, TH* d_h, TF* d_f, float* parts)
{
    constexpr int kAhead = WIDE || R > 1 ? 1 : 2;
    __shared__ float lds[WIDE ? 2 * 16 : kThreads / 64 * kWaveChannels];
    const Group<WIDE> g(d, lds);
    float post_gamma[R * V], gate[R * V], gamma[R * V];
    parameter<WHOLE, V, R>(d, g, d.post_gamma, 1.0f, post_gamma);
    parameter<WHOLE, V, R>(d, g, d.gamma, 1.0f, gamma);
    const long long items = d.N * d.chunks;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long n = item / d.chunks, first = (item - n * d.chunks) * d.chunk, end = min(d.P, first + d.chunk);
        parameter<WHOLE, V, R>(d, g, d.gate ? d.gate + n * d.C : nullptr, 1.0f, gate);
        float sums[3][R * V];
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int e = 0; e < R * V; ++e) sums[k][e] = 0.0f;
        Pack<TH, V> hp[R], dsp[R], h_next[kAhead][R], ds_next[kAhead][R];
        Pack<TF, V> fp[R], dyp[R], f_next[kAhead][R], dy_next[kAhead][R];
        const long long start = n * d.P + first + g.index, mine = first + g.index;
        const TH *h_at = h + start * d.hs, *ds_at = d_s + start * d.hs;
        const TF *f_at = f + start * d.fs, *dy_at = d_y + start * d.ys;
        TH* dh_at = d_h + start * d.hs;
        TF* df_at = d_f + start * d.fs;
        auto ask = [&](long long p, int u) {
            if (p < end) {
                if (d_y) {
                    load<WHOLE, TH, V, R>(d, g, h_at, h_next[u]);
                    load<WHOLE, TF, V, R>(d, g, dy_at, dy_next[u]);
                }
                if (f) load<WHOLE, TF, V, R>(d, g, f_at, f_next[u]);
                if (d_s) load<WHOLE, TH, V, R>(d, g, ds_at, ds_next[u]);
            }
            h_at += d.groups * d.hs;
            ds_at += d.groups * d.hs;
            f_at += d.groups * d.fs;
            dy_at += d.groups * d.ys;
        };
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ask(mine + u * d.groups, u);
        for (long long p = mine; p < end; p += d.groups) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                hp[r] = h_next[0][r];
                fp[r] = f_next[0][r];
                dsp[r] = ds_next[0][r];
                dyp[r] = dy_next[0][r];
#pragma unroll
                for (int u = 1; u < kAhead; ++u) {
                    h_next[u - 1][r] = h_next[u][r];
                    f_next[u - 1][r] = f_next[u][r];
                    ds_next[u - 1][r] = ds_next[u][r];
                    dy_next[u - 1][r] = dy_next[u][r];
                }
            }
            ask(p + kAhead * d.groups, kAhead - 1);
            float fh[R * V], grad[R * V], rstd_f = 1.0f;
            if (f) {
                widen<WHOLE, TF, V, R>(d, g, fp, fh);
                if (d.post) rstd_f = normalise<WHOLE, V, R>(d, g, fh);
            }
            if (d_y) {
                float t[R * V];
                widen<WHOLE, TH, V, R>(d, g, hp, t);
                if (f) {
#pragma unroll
                    for (int e = 0; e < R * V; ++e) t[e] = fmaf(gate[e], d.post ? post_gamma[e] * fh[e] : fh[e], d.alpha * t[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < R * V; ++e) t[e] *= d.alpha;
                }
                const float rstd = normalise<WHOLE, V, R>(d, g, t);
                widen<WHOLE, TF, V, R>(d, g, dyp, grad);
#pragma unroll
                for (int e = 0; e < R * V; ++e) {
                    sums[0][e] = fmaf(grad[e], t[e], sums[0][e]);
                    sums[1][e] += grad[e];
                    grad[e] *= gamma[e];
                }
                normalise_grad<V, R>(d, g, t, rstd, grad);
            } else {
#pragma unroll
                for (int e = 0; e < R * V; ++e) grad[e] = 0.0f;
            }
            if (d_s) {
                float up[R * V];
                widen<WHOLE, TH, V, R>(d, g, dsp, up);
#pragma unroll
                for (int e = 0; e < R * V; ++e) grad[e] += up[e];
            }
            if (d_h) {
                float r[R * V];
#pragma unroll
                for (int e = 0; e < R * V; ++e) r[e] = d.alpha * grad[e];
                store<WHOLE, TH, V, R>(d, g, dh_at, r);
                dh_at += d.groups * d.hs;
            }
            if (!f) continue;
#pragma unroll
            for (int e = 0; e < R * V; ++e) sums[2][e] = fmaf(grad[e], fh[e], sums[2][e]);
            if (!d_f) continue;
#pragma unroll
            for (int e = 0; e < R * V; ++e) grad[e] *= d.post ? gate[e] * post_gamma[e] : gate[e];
            if (d.post) normalise_grad<V, R>(d, g, fh, rstd_f, grad);
            store<WHOLE, TF, V, R>(d, g, df_at, grad);
            df_at += d.groups * d.fs;
        }
        if (!parts) continue;
        float* part = parts + item * 3 * d.C;
        if (WIDE) {
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int c = (r * g.lanes + g.lane) * V;
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (on<WHOLE, V>(d, g, r, j)) part[k * d.C + c + j] = sums[k][r * V + j];
                }
        } else {
            const int wave = threadIdx.x >> 6;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                // first the groups of a wave, then the waves
                for (int m = d.lanes; m < 64; m <<= 1)
#pragma unroll
                    for (int e = 0; e < R * V; ++e) sums[k][e] += __shfl_xor(sums[k][e], m);
                __syncthreads();   // (the sums before have been read)
                if ((threadIdx.x & 63) < d.lanes)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int c = (r * g.lanes + g.lane) * V;
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            if (on<WHOLE, V>(d, g, r, j)) lds[wave * kWaveChannels + c + j] = sums[k][r * V + j];
                    }
                __syncthreads();
                for (int c = threadIdx.x; c < d.C; c += kThreads) {
                    float sum = lds[c];
#pragma unroll
                    for (int w = 1; w < kThreads / 64; ++w) sum += lds[w * kWaveChannels + c];
                    part[k * d.C + c] = sum;
                }
            }
        }
    }
}

// Columns' sums over `n` rows `stride` apart, of kJoinColumns columns: thread (row lane, column); the result is in row lane 0.
constexpr int kJoinColumns = 16;
__device__ __forceinline__ double column_sum(const float* at, long long n, long long stride, bool in, double* lds)
{
    constexpr int kRows = kJoinThreads / kJoinColumns;
    const int row = threadIdx.x / kJoinColumns;
    double sum = 0.0;
    if (in) {
#pragma unroll 8
        for (long long i = row; i < n; i += kRows) sum += (double)at[i * stride];
    }
    // the rows of a wave, then the waves
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    __syncthreads();
    if ((threadIdx.x & 63) < kJoinColumns) lds[(threadIdx.x >> 6) * kJoinColumns + (threadIdx.x & 63)] = sum;
    __syncthreads();
    if (row) return 0.0;
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) sum += lds[w * kJoinColumns + threadIdx.x];
    return sum;
}

// Workgroup (kJoinColumns columns; y = 0: d_gamma, 1: d_beta, from 2 on: the samples' T).  T goes to the gate, and to the post norm's gradient
// where there is one sample, else as gate T into `terms` [N][C] for the kernel below.
__global__ __launch_bounds__(kJoinThreads) void residual_norm_join_kernel(NormDev d, const float* parts, float* d_gamma, float* d_beta,
                                                                         float* d_post_gamma, float* d_gate, float* terms)
{
    __shared__ double lds[kJoinThreads / 64 * kJoinColumns];
    const int c = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    const bool in = c < d.C, first = threadIdx.x < kJoinColumns;
    const long long row = 3ll * d.C;
    if (blockIdx.y < 2) {
        float* out = blockIdx.y ? d_beta : d_gamma;
        if (!out) return;
        const double sum = column_sum(parts + blockIdx.y * (long long)d.C + c, d.N * d.chunks, row, in, lds);
        if (in && first) out[c] += (float)sum;
        return;
    }
    if (!d_gate && !d_post_gamma) return;
    for (long long n = blockIdx.y - 2; n < d.N; n += gridDim.y - 2) {
        const double sum = column_sum(parts + n * d.chunks * row + 2ll * d.C + c, d.chunks, row, in, lds);
        if (!in || !first) continue;
        if (d_gate) d_gate[n * d.C + c] += (float)(d.post && d.post_gamma ? sum * d.post_gamma[c] : sum);
        const float term = (float)(d.gate ? sum * d.gate[n * d.C + c] : sum);
        if (terms) terms[n * d.C + c] = term;
        else if (d_post_gamma) d_post_gamma[c] += term;
    }
}
__global__ __launch_bounds__(kJoinThreads) void residual_norm_terms_kernel(NormDev d, const float* terms, float* d_post_gamma)
{
    __shared__ double lds[kJoinThreads / 64 * kJoinColumns];
    const int c = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    const double sum = column_sum(terms + c, d.N, d.C, c < d.C, lds);
    if (c < d.C && threadIdx.x < kJoinColumns) d_post_gamma[c] += (float)sum;
}

// ---- host ------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int dtype_bytes(int t) { return t == LP_F32 ? 4 : 2; }

lp_status validate(const lp_residual_norm* q, NormDev* d)
{
    if (!q) return fail(LP_ERR_INVALID_ARG, "norm must not be NULL");
    if (q->N < 0 || q->P < 0) return fail(LP_ERR_INVALID_ARG, "norm->N and norm->P must be >= 0");
    if (q->C < 1) return fail(LP_ERR_INVALID_ARG, "norm->C must be >= 1");
    if (q->C > LP_RESIDUAL_NORM_MAX_CHANNELS) return fail(LP_ERR_UNSUPPORTED, "norm->C is beyond LP_RESIDUAL_NORM_MAX_CHANNELS");
    if (q->kind != LP_NORM_RMS && q->kind != LP_NORM_LAYER) return fail(LP_ERR_INVALID_ARG, "norm->kind must be an lp_norm_kind");
    if ((q->post_norm | q->gate_per_sample) & ~1) return fail(LP_ERR_INVALID_ARG, "norm->post_norm and norm->gate_per_sample must be 0 or 1");
    if (!std::isfinite(q->eps) || q->eps < 0.0f) return fail(LP_ERR_INVALID_ARG, "norm->eps must be finite and >= 0");
    if (!std::isfinite(q->alpha)) return fail(LP_ERR_INVALID_ARG, "norm->alpha must be finite");
    for (int t : {q->h_dtype, q->f_dtype})
        if (t != LP_F32 && t != LP_BF16 && t != LP_F16)
            return fail(LP_ERR_INVALID_ARG, "norm->h_dtype and norm->f_dtype must be LP_F32, LP_BF16 or LP_F16");
    if (q->h_dtype != q->f_dtype && q->h_dtype != LP_F32)
        return fail(LP_ERR_UNSUPPORTED, "norm->f_dtype must be norm->h_dtype unless that is LP_F32");
    if (q->post_gamma && !q->post_norm) return fail(LP_ERR_INVALID_ARG, "norm->post_gamma needs norm->post_norm");
    std::memset(d, 0, sizeof(*d));
    double most = 0.0;
    const int64_t strides[3] = {q->h_stride, q->f_stride, q->y_stride};
    long long* to[3] = {&d->hs, &d->fs, &d->ys};
    for (int k = 0; k < 3; ++k) {
        *to[k] = strides[k] ? strides[k] : q->C;
        if (*to[k] < q->C) return fail(LP_ERR_INVALID_ARG, "norm's strides must be 0 or >= norm->C");
        most = std::fmax(most, (double)*to[k]);
    }
    if ((double)q->N * (double)q->P * most * 4.0 > 4e18) return fail(LP_ERR_UNSUPPORTED, "norm: tensors beyond 64-bit offsets");
    d->N = q->N; d->P = q->P;
    d->C = q->C; d->layer = q->kind == LP_NORM_LAYER; d->post = q->post_norm; d->eps = q->eps; d->alpha = q->alpha;
    d->post_gamma = q->post_gamma; d->gate = q->gate; d->gamma = q->gamma; d->beta = q->beta;
    if (!q->gate_per_sample) {   // positions are all alike
        d->P *= d->N;
        d->N = d->P ? 1 : 0;
    }
    return LP_OK;
}

// Divides the samples among some workgroups a compute unit, at least four positions a group; what the backward's workspace has room for
// is counted with the fewest positions at a time.
void divide(NormDev* d, int n_cu, int per_cu)
{
    const long long target = (long long)per_cu * n_cu / (d->N > 0 ? d->N : 1), most = (d->P + 4ll * d->groups - 1) / (4ll * d->groups);
    long long chunks = target < most ? target : most;
    if (chunks < 1) chunks = 1;
    d->chunk = (d->P + chunks - 1) / chunks;
    if (d->chunk < 1) d->chunk = 1;
    d->chunks = (int)((d->P + d->chunk - 1) / d->chunk);
    if (d->chunks < 1) d->chunks = 1;
}

struct Shape {
    int V, R;
    bool wide, whole;
    unsigned threads;
};

// Lanes and slots of a position: few idle lanes first, then few slots.
Shape shape(NormDev* d, int V)
{
    Shape s = {V, 1, false, d->C % V == 0, kThreads};
    const int slots = (d->C + V - 1) / V;
    if (d->C > kWaveChannels) {
        s.wide = true;
        s.R = (d->C > kWideThreads * kHeld ? 2 * kHeld : kHeld) / V;
        const int waves = (slots + 64 * s.R - 1) / (64 * s.R);
        s.threads = 64 * waves;
        d->lanes = 64 * waves;
        d->groups = 1;
        return s;
    }
    int best = 0;
    for (int R = 1; R <= kHeld / V; R *= 2) {
        int lanes = 1;
        while (lanes * R < slots) lanes *= 2;
        if (lanes > 64) continue;
        if (!best || lanes * R < best) {
            best = lanes * R;
            s.R = R;
            d->lanes = lanes;
        }
    }
    d->groups = kThreads / d->lanes;
    return s;
}

// Workgroups a compute unit, as many as its registers hold at once: a few more would run alone at the end (24 x 256^2 x 32, gradients: 4 take
// 202 us, 3 and 6 take 213 and 223, 43 for each of the 24 samples, 1032 on 1024 places, 285).  With eight channels a lane the gradients' kernel has
// room for three, but two are faster (65536 x 512 in bf16: 101 us, three 106).
constexpr int kForwardPerUnit = 5;
int backward_per_unit(const Shape& s) { return s.R * s.V >= kHeld ? 2 : 4; }

struct Sizes {
    size_t parts, terms;
};
Sizes sizes(const NormDev& d, int V, int n_cu)
{
    NormDev t = d;
    const Shape shp = shape(&t, V);
    divide(&t, n_cu, backward_per_unit(shp));
    const long long items = t.N * t.chunks;
    return {align256((size_t)items * 3 * d.C * sizeof(float)), d.post && d.N > 1 ? align256((size_t)d.N * d.C * sizeof(float)) : 0};
}

int slot_width(const lp_residual_norm* q) { return 16 / dtype_bytes(q->h_dtype); }   // 16 bytes of h

// Calls f with the types, the slots' width and number and whether a position takes a workgroup as constants.
template <class T> struct Type { using type = T; };
template <class F, class H, class B>
void with_shape(const Shape& s, F&& f, Type<H> h, Type<B> b)
{
    constexpr int W = 16 / sizeof(H);
    auto one = [&](auto r) {
        if (s.R != r.value) return;
        constexpr int held = W * decltype(r)::value;
        auto v = std::integral_constant<int, W>();
        auto go = [&](auto wide) { s.whole ? f(h, b, v, r, wide, std::true_type()) : f(h, b, v, r, wide, std::false_type()); };
        if constexpr (held >= kHeld) {
            if (s.wide) go(std::true_type());
        }
        if constexpr (held <= kHeld) {
            if (!s.wide) go(std::false_type());
        }
    };
    one(std::integral_constant<int, 1>());
    one(std::integral_constant<int, 2>());
    if constexpr (W == 4) one(std::integral_constant<int, 4>());
}
template <class F>
void dispatch(int h_dtype, int f_dtype, const Shape& s, F&& f)
{
    if (h_dtype == LP_BF16) with_shape(s, f, Type<__bf16>(), Type<__bf16>());
    else if (h_dtype == LP_F16) with_shape(s, f, Type<_Float16>(), Type<_Float16>());
    else if (f_dtype == LP_BF16) with_shape(s, f, Type<float>(), Type<__bf16>());
    else if (f_dtype == LP_F16) with_shape(s, f, Type<float>(), Type<_Float16>());
    else with_shape(s, f, Type<float>(), Type<float>());
}

// Bytes that a call moves of tensors like h and like f.
double bytes_of(const lp_residual_norm* q, int hs, int fs)
{
    return (double)q->N * (double)q->P * q->C * (hs * dtype_bytes(q->h_dtype) + fs * dtype_bytes(q->f_dtype));
}

unsigned grid_of(long long items) { return (unsigned)(items < kMaxGrid ? items : kMaxGrid); }

lp_status launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LP_OK : fail(LP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

lp_status aligned(const lp_residual_norm* q, std::initializer_list<const void*> hs, std::initializer_list<const void*> fs)
{
    for (const void* p : hs)
        if ((uintptr_t)p % dtype_bytes(q->h_dtype)) return fail(LP_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    for (const void* p : fs)
        if ((uintptr_t)p % dtype_bytes(q->f_dtype)) return fail(LP_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    return LP_OK;
}

lp_status forward(const lp_residual_norm* q, const void* h, const void* f, void* s, void* y, hipStream_t stream)
{
    NormDev d;
    lp_status st = validate(q, &d);
    if (st != LP_OK) return st;
    if (d.N == 0 || d.P == 0 || (!s && !y)) return LP_OK;
    if (!h) return fail(LP_ERR_INVALID_ARG, "h must not be NULL");
    if ((st = aligned(q, {h, s}, {f, y})) != LP_OK) return st;
    std::string err;
    int n_cu = 0;
    if (compute_units(&n_cu, &err)) return fail(LP_ERR_HIP, err);
    const Shape shp = shape(&d, slot_width(q));
    divide(&d, n_cu, kForwardPerUnit);
    d.past_cache = bytes_of(q, 1 + (s != nullptr), (f != nullptr) + (y != nullptr)) > kCacheBytes;
    dispatch(q->h_dtype, q->f_dtype, shp, [&](auto th, auto tf, auto v, auto r, auto wide, auto whole) {
        using TH = typename decltype(th)::type;
        using TF = typename decltype(tf)::type;
        hipLaunchKernelGGL((residual_norm_kernel<TH, TF, decltype(v)::value, decltype(r)::value, decltype(wide)::value, decltype(whole)::value>),
                           dim3(grid_of(d.N * d.chunks)), dim3(shp.threads), 0, stream, d, (const TH*)h, (const TF*)f, (TH*)s, (TF*)y);
    });
    return launched("residual norm forward launch");
}

lp_status backward(const lp_residual_norm* q, const void* h, const void* f, const void* d_s, const void* d_y, void* d_h, void* d_f,
                   float* d_gamma, float* d_beta, float* d_post_gamma, float* d_gate, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    NormDev d;
    lp_status st = validate(q, &d);
    if (st != LP_OK) return st;
    if (d.N == 0 || d.P == 0) return LP_OK;
    if (!h) return fail(LP_ERR_INVALID_ARG, "h must not be NULL");
    if (!f && (d_f || d_post_gamma || d_gate)) return fail(LP_ERR_INVALID_ARG, "d_f, d_post_gamma and d_gate need f");
    if (d_post_gamma && !d.post) return fail(LP_ERR_INVALID_ARG, "d_post_gamma needs norm->post_norm");
    if ((st = aligned(q, {h, d_s, d_h}, {f, d_y, d_f})) != LP_OK) return st;
    std::string err;
    int n_cu = 0;
    if (compute_units(&n_cu, &err)) return fail(LP_ERR_HIP, err);
    const Sizes size = sizes(d, slot_width(q), n_cu);
    if (!workspace || workspace_bytes < size.parts + size.terms)
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_residual_norm_workspace_bytes");
    if ((uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const Shape shp = shape(&d, slot_width(q));
    divide(&d, n_cu, backward_per_unit(shp));
    d.past_cache = bytes_of(q, 1 + (d_s != nullptr) + (d_h != nullptr), (f != nullptr) + (d_y != nullptr) + (d_f != nullptr)) > kCacheBytes;
    const bool sums = d_gamma || d_beta || d_post_gamma || d_gate;
    if (!sums && !d_h && !d_f) return LP_OK;
    float* parts = sums ? (float*)workspace : nullptr;
    float* terms = d.N > 1 && d_post_gamma ? (float*)((char*)workspace + size.parts) : nullptr;
    dispatch(q->h_dtype, q->f_dtype, shp, [&](auto th, auto tf, auto v, auto r, auto wide, auto whole) {
        using TH = typename decltype(th)::type;
        using TF = typename decltype(tf)::type;
        hipLaunchKernelGGL((residual_norm_grad_kernel<TH, TF, decltype(v)::value, decltype(r)::value, decltype(wide)::value, decltype(whole)::value>),
                           dim3(grid_of(d.N * d.chunks)), dim3(shp.threads), 0, stream, d, (const TH*)h, (const TF*)f, (const TH*)d_s,
                           (const TF*)d_y, (TH*)d_h, (TF*)d_f, parts);
    });
    if (sums) {
        const dim3 grid((d.C + kJoinColumns - 1) / kJoinColumns, 2 + (unsigned)(d.N < 4096 ? d.N : 4096));
        hipLaunchKernelGGL(residual_norm_join_kernel, grid, dim3(kJoinThreads), 0, stream, d, parts, d_gamma, d_beta, d_post_gamma, d_gate, terms);
        if (terms) hipLaunchKernelGGL(residual_norm_terms_kernel, dim3(grid.x), dim3(kJoinThreads), 0, stream, d, terms, d_post_gamma);
    }
    return launched("residual norm backward launch");
}

}  // namespace

}  // namespace lp

extern "C" {

lp_status lp_residual_norm_workspace_bytes(const lp_residual_norm* norm, size_t* bwd_bytes)
try {
    lp::NormDev d;
    const lp_status st = lp::validate(norm, &d);
    if (st != LP_OK) return st;
    if (!bwd_bytes) return lp::fail(LP_ERR_INVALID_ARG, "bwd_bytes must not be NULL");
    std::string err;
    int n_cu = 0;
    if (lp::compute_units(&n_cu, &err)) return lp::fail(LP_ERR_HIP, err);
    const lp::Sizes size = lp::sizes(d, lp::slot_width(norm), n_cu);
    *bwd_bytes = size.parts + size.terms;
    return LP_OK;
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_residual_norm_fwd(const lp_residual_norm* norm, const void* h, const void* f, void* s, void* y, void* stream)
try {
    return lp::forward(norm, h, f, s, y, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_residual_norm_bwd(const lp_residual_norm* norm, const void* h, const void* f, const void* d_s, const void* d_y, void* d_h,
                               void* d_f, float* d_gamma, float* d_beta, float* d_post_gamma, float* d_gate, void* workspace,
                               size_t workspace_bytes, void* stream)
try {
    return lp::backward(norm, h, f, d_s, d_y, d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

}  // extern "C"
