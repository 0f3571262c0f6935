// Products of positions' channels with a weight matrix, with bias, activation and residual in the epilogue, and their gradients.
//
//     z = x W^T + b,   y = act(z) + r;   d_z = d_y act'(z),   d_x = d_z W,   d_W += d_z^T x,   d_b += sum d_z
//
// What bounds it: memory where a grid's positions have few channels (32 -> 64 channels in fp32: 380 bytes for 4096 operations a position), the
// matrix cores for blocks of some hundred channels, latency for single tokens.
//
// Everything moves in chunks of 16 bytes along the channels.  A 32 x 32 block of results is made from chunks the same way in all types: of two
// neighbouring chunks of a row lanes 0 .. 31 hold the first, lanes 32 .. 63 the second, and that is one 32x32x16 product in 16 bits and
// four 32x32x2 products in fp32 (the order of the channels in a sum does not matter as long as both operands have the same).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "lp_act.h"
#include "lp_kernels.h"

namespace lp {

using namespace act;

namespace {

constexpr int kThreads = 256;
constexpr unsigned kMaxGrid = 1u << 30;
constexpr int kFewRows = 8;   // positions that go to the kernel without matrix cores, at most

using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));

template <class T> struct Vec;
template <> struct Vec<float> { using Of = float __attribute__((ext_vector_type(4))); };
template <> struct Vec<__bf16> { using Of = __bf16 __attribute__((ext_vector_type(8))); };
template <> struct Vec<_Float16> { using Of = _Float16 __attribute__((ext_vector_type(8))); };

// 16 bytes of neighbouring channels.
template <class T>
struct alignas(16) Chunk {
    static constexpr int kCount = 16 / sizeof(T);
    T v[kCount];
};
template <class T> constexpr int kChunk = Chunk<T>::kCount;

// `count` (may be <= 0) values from p, zeros behind them.  A whole chunk is one load, also where it is not aligned to 16 bytes.
template <class T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, long long count)
{
    Chunk<T> c;
    if (count >= kChunk<T>) {
        __builtin_memcpy(&c, p, 16);
    } else {
#pragma unroll
        for (int j = 0; j < kChunk<T>; ++j) c.v[j] = j < count ? p[j] : (T)0.0f;
    }
    return c;
}
template <class T>
__device__ __forceinline__ void store_chunk(T* p, long long count, const Chunk<T>& c)
{
    if (count >= kChunk<T>) {
        __builtin_memcpy(p, &c, 16);
    } else {
#pragma unroll
        for (int j = 0; j < kChunk<T>; ++j)
            if (j < count) p[j] = c.v[j];
    }
}

// acc += a b^T over the channels of two neighbouring chunks (see above)
__device__ __forceinline__ f32x16 multiply(const Chunk<__bf16>& a, const Chunk<__bf16>& b, f32x16 acc)
{
    using V = Vec<__bf16>::Of;
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(const Chunk<_Float16>& a, const Chunk<_Float16>& b, f32x16 acc)
{
    using V = Vec<_Float16>::Of;
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(const Chunk<float>& a, const Chunk<float>& b, f32x16 acc)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], acc, 0, 0, 0);
    return acc;
}

// d_z of a chunk, rounded to T, and what the rounding left.
template <class T>
struct Gradient {
    Chunk<T> hi, lo;
    float v[kChunk<T>];
};
template <int ACT, class T>
__device__ __forceinline__ Gradient<T> gradient(const Chunk<T>& dy, const Chunk<T>& pre)
{
    Gradient<T> g;
#pragma unroll
    for (int j = 0; j < kChunk<T>; ++j) {
        g.v[j] = (float)dy.v[j] * (ACT == LP_ACT_NONE ? 1.0f : slope<ACT>((float)pre.v[j]));
        asm("" : "+v"(g.v[j]));   // (both parts come from this value: hi alone could be rounded straight from the product)
        g.hi.v[j] = (T)g.v[j];
        if (sizeof(T) == 2) {
            const float rest = g.v[j] - (float)g.hi.v[j];
            g.lo.v[j] = (T)(__builtin_isfinite(rest) ? rest : 0.0f);   // (of an infinite d_z nothing is left)
        }
    }
    return g;
}

struct LinearDev {
    long long P;
    int K, N;                       // of the product: channels that are summed over, channels of the result
    long long as, ys, rs;           // elements from position to position: operand, result, residual
    const void *a, *w, *res, *pre;  // w: [N][ws]; pre (of the backward): [P][K]
    long long ws;
    const float* bias;
    void *out, *keep;               // keep: [P][N]
    long long tiles_p;
    int tiles_n;
};

// ---- tiles -----------------------------------------------------------------------------------------------------
//
// A workgroup of four waves makes BP positions x BN channels.  A step is 128 bytes of channels of both operands, staged through
// registers into one of two LDS buffers while the other one is multiplied.  A row's eight chunks lie at chunk ^ (row mod 8): eight
// rows' same chunk, and a row's eight chunks, both touch every bank once.
template <int BP, int BN>
struct TileShape {
    static constexpr int kWavesN = BN >= 128 ? 2 : 1, kWavesP = 4 / kWavesN;
    static constexpr int kP = BP / kWavesP, kN = BN / kWavesN;          // of a wave
    static constexpr int kBlocksP = kP / 32, kBlocksN = kN / 32;
    static constexpr int kPitch = kN + 4;                               // floats of a position's row while results are turned over
    static constexpr int kStage = (BP + BN) * 128;                      // bytes of a step
    static constexpr int kLds = 2 * kStage > 4 * 32 * kPitch * 4 ? 2 * kStage : 4 * 32 * kPitch * 4;
};

__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * 128 + ((chunk ^ (row & 7)) << 4); }

// Tile of a workgroup: neighbouring workgroups go to the chip's eight XCDs in turn, so each of these takes one run of the
// tiles; channels' tiles of the same positions follow one another (their positions are read from the XCD's L2).
__device__ __forceinline__ long long tile_of(long long b, long long tiles)
{
    const long long each = (tiles + 7) / 8;
    return (b & 7) * each + (b >> 3);
}

template <class T, int ACT, bool BACK, int BP, int BN>
__global__ __launch_bounds__(kThreads, 2) void linear_tile_kernel(LinearDev d)
{
    using S = TileShape<BP, BN>;
    constexpr int E = kChunk<T>;
    constexpr int kLoadsA = BP * 8 / kThreads, kLoadsW = BN * 8 / kThreads;
    __shared__ alignas(16) char lds[S::kLds];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
    const int wave_p = wave / S::kWavesN * S::kP, wave_n = wave % S::kWavesN * S::kN;
    const int c8 = threadIdx.x & 7, row = threadIdx.x >> 3;
    const long long tiles = d.tiles_p * d.tiles_n, rounds = (tiles + 7) / 8 * 8;
    for (long long b = blockIdx.x; b < rounds; b += gridDim.x) {
        const long long tile = tile_of(b, tiles);
        if (tile >= tiles) continue;
        const long long p0 = tile / d.tiles_n * BP;
        const int n0 = (int)(tile % d.tiles_n) * BN;
        Chunk<T> a[kLoadsA], pre[BACK && ACT != LP_ACT_NONE ? kLoadsA : 1], w[kLoadsW];
        auto ask = [&](int k0) {
            const int k = k0 + c8 * E;
#pragma unroll
            for (int u = 0; u < kLoadsA; ++u) {
                const long long p = p0 + row + u * 32;
                const int count = p < d.P ? d.K - k : 0;
                a[u] = load_chunk((const T*)d.a + p * d.as + k, count);
                if (BACK && ACT != LP_ACT_NONE) pre[u] = load_chunk((const T*)d.pre + p * d.K + k, count);
            }
#pragma unroll
            for (int u = 0; u < kLoadsW; ++u) {
                const int n = n0 + row + u * 32;
                w[u] = load_chunk((const T*)d.w + n * d.ws + k, n < d.N ? d.K - k : 0);
            }
        };
        auto put = [&](int buffer) {
            char* to = lds + buffer * S::kStage;
#pragma unroll
            for (int u = 0; u < kLoadsA; ++u) {
                Chunk<T> v = a[u];
                if (BACK && ACT != LP_ACT_NONE) v = gradient<ACT>(a[u], pre[u]).hi;
                *(Chunk<T>*)(to + chunk_at(row + u * 32, c8)) = v;
            }
#pragma unroll
            for (int u = 0; u < kLoadsW; ++u) *(Chunk<T>*)(to + BP * 128 + chunk_at(row + u * 32, c8)) = w[u];
        };
        f32x16 acc[S::kBlocksN][S::kBlocksP] = {};
        const int steps = (d.K + 8 * E - 1) / (8 * E);
        ask(0);
        put(0);
        __syncthreads();
        for (int s = 0; s < steps; ++s) {
            if (s + 1 < steps) ask((s + 1) * 8 * E);
            const char* from = lds + (s & 1) * S::kStage;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                Chunk<T> wv[S::kBlocksN], av[S::kBlocksP];
#pragma unroll
                for (int i = 0; i < S::kBlocksN; ++i) wv[i] = *(const Chunk<T>*)(from + BP * 128 + chunk_at(wave_n + i * 32 + l32, 2 * q + h));
#pragma unroll
                for (int i = 0; i < S::kBlocksP; ++i) av[i] = *(const Chunk<T>*)(from + chunk_at(wave_p + i * 32 + l32, 2 * q + h));
#pragma unroll
                for (int i = 0; i < S::kBlocksN; ++i)
#pragma unroll
                    for (int j = 0; j < S::kBlocksP; ++j) acc[i][j] = multiply(wv[i], av[j], acc[i][j]);
            }
            if (s + 1 < steps) put((s + 1) & 1);
            __syncthreads();
        }
        // Results: value e of a lane is channel 8 (e / 4) + 4 h + e % 4 of position l32 of a block.  They are turned over in the wave's
        // own LDS, so that neighbouring lanes write neighbouring channels.
        float* turn = (float*)lds + wave * 32 * S::kPitch;
        constexpr int kAcross = S::kN / E, kDown = 64 / kAcross;   // lanes of a position, positions at a time
        const int n = n0 + wave_n + lane % kAcross * E;
        float bias[E];
#pragma unroll
        for (int j = 0; j < E; ++j) bias[j] = d.bias && n + j < d.N ? d.bias[n + j] : 0.0f;
#pragma unroll
        for (int jp = 0; jp < S::kBlocksP; ++jp) {
#pragma unroll
            for (int i = 0; i < S::kBlocksN; ++i)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *(f32x4*)(turn + l32 * S::kPitch + i * 32 + 2 * e + 4 * h) = f32x4{acc[i][jp][e], acc[i][jp][e + 1], acc[i][jp][e + 2], acc[i][jp][e + 3]};
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int r = 0; r < 32 / kDown; ++r) {
                const int at = r * kDown + lane / kAcross;
                const long long p = p0 + wave_p + jp * 32 + at;
                const int count = p < d.P ? d.N - n : 0;
                float z[E];
#pragma unroll
                for (int j = 0; j < E; j += 4) *(f32x4*)(z + j) = *(const f32x4*)(turn + at * S::kPitch + lane % kAcross * E + j);
                Chunk<T> out;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    z[j] += bias[j];
                    out.v[j] = (T)z[j];
                }
                if (!BACK) {
                    if (d.keep) store_chunk((T*)d.keep + p * d.N + n, count, out);
                    Chunk<T> res = {};
                    if (d.res) res = load_chunk((const T*)d.res + p * d.rs + n, count);
#pragma unroll
                    for (int j = 0; j < E; ++j) out.v[j] = (T)(activate<ACT>(z[j]) + (float)res.v[j]);
                }
                store_chunk((T*)d.out + p * d.ys + n, count, out);
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();   // (the next tile's first step lies where results were)
    }
}

// ---- few positions ---------------------------------------------------------------------------------------------
//
// A wave makes kOutputs channels of up to ROWS positions: lanes share the sum, 16 bytes of a weight's row each.
constexpr int kOutputs = 2;
template <class T, int ACT, int ROWS>
__global__ __launch_bounds__(kThreads) void linear_rows_kernel(LinearDev d)
{
    constexpr int E = kChunk<T>;
    const int lane = threadIdx.x & 63, n0 = (blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * kOutputs;
    if (n0 >= d.N) return;
    float sum[kOutputs][ROWS] = {};
    for (int k = lane * E; k < d.K; k += 64 * E) {
        Chunk<T> w[kOutputs], x[ROWS];
#pragma unroll
        for (int i = 0; i < kOutputs; ++i) w[i] = load_chunk((const T*)d.w + (n0 + i) * d.ws + k, n0 + i < d.N ? d.K - k : 0);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) x[r] = load_chunk((const T*)d.a + r * d.as + k, r < d.P ? d.K - k : 0);
#pragma unroll
        for (int i = 0; i < kOutputs; ++i)
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int j = 0; j < E; ++j) sum[i][r] = fmaf((float)w[i].v[j], (float)x[r].v[j], sum[i][r]);
    }
#pragma unroll
    for (int m = 32; m; m >>= 1)
#pragma unroll
        for (int i = 0; i < kOutputs; ++i)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) sum[i][r] += __shfl_xor(sum[i][r], m);
#pragma unroll
    for (int i = 0; i < kOutputs; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int n = n0 + i;
            if (lane != i * ROWS + r || n >= d.N || r >= d.P) continue;
            const float z = sum[i][r] + (d.bias ? d.bias[n] : 0.0f);
            if (d.keep) ((T*)d.keep)[(long long)r * d.N + n] = (T)z;
            float y = activate<ACT>(z);
            if (d.res) y += (float)((const T*)d.res)[r * d.rs + n];
            ((T*)d.out)[r * d.ys + n] = (T)y;
        }
}

// ---- gradients of the parameters -------------------------------------------------------------------------------
//
// A workgroup sums a part of the positions into 128 channels of d_z x 128 channels of x.  The sum runs over the rows as they
// lie in memory, so in 16 bits the operands come from LDS by the transposing read (16 lanes point at the 8-byte quarters of 4 rows x 16
// columns and receive a column each).  A row has 64 bytes more than its channels: four rows' quarters touch every bank once.
struct WeightDev {
    long long P;
    int K, N;
    long long xs, ys;
    const void *x, *dy, *pre;
    float *d_weight, *d_bias;
    float *parts, *bias_parts;   // [splits][N][K], [splits][N]; NULL: one split, into d_weight and d_bias
    long long chunk;             // positions of a part
    int tiles_n, tiles_k, splits;
};
constexpr int kWeightTile = 128;

template <class T> constexpr int kWeightPitch = kWeightTile * sizeof(T) + 64;   // bytes
template <class T> constexpr int kWeightRows = 32;

__device__ __forceinline__ u32x2 read_transposed(const char* at)
{
    typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4 Lds;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)at));
}

// 32 columns from `column` on over rows r0 .. r0 + 15, as an operand (element e of a lane of half h: row 8 (e / 4) + 4 h + e % 4)
template <class T>
__device__ __forceinline__ Chunk<T> columns(const char* image, int r0, int column, int lane)
{
    const int q = lane >> 4, t = lane & 15;
    const char* at = image + (r0 + 4 * (q >> 1) + (t >> 2)) * kWeightPitch<T> + (column + 16 * (q & 1) + 4 * (t & 3)) * 2;
    const u32x2 a = read_transposed(at), b = read_transposed(at + 8 * kWeightPitch<T>);
    return __builtin_bit_cast(Chunk<T>, u32x4{a[0], a[1], b[0], b[1]});
}

template <class T, int ACT>
__global__ __launch_bounds__(kThreads, 2) void linear_weight_kernel(WeightDev d)
{
    constexpr int E = kChunk<T>, kRows = kWeightRows<T>, kPitch = kWeightPitch<T>;
    constexpr bool kSplit = sizeof(T) == 2 && ACT != LP_ACT_NONE;   // d_z in two parts
    constexpr int kAcross = kWeightTile / E, kDown = kThreads / kAcross, kLoads = kRows / kDown;
    constexpr int kImage = kRows * kPitch, kStage = kImage * (kSplit ? 3 : 2);
    __shared__ alignas(16) char lds[2 * kStage];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
    const int c = threadIdx.x % kAcross, row = threadIdx.x / kAcross;
    const int wave_n = (wave >> 1) * 64, wave_k = (wave & 1) * 64;
    const int tiles = d.tiles_n * d.tiles_k, split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int n0 = tile / d.tiles_k * kWeightTile, k0 = tile % d.tiles_k * kWeightTile;
    const long long first = split * d.chunk, end = min(d.P, first + d.chunk);
    Chunk<T> dy[kLoads], pre[kLoads], x[kLoads];
    float bias[E] = {};
    const int n = n0 + c * E, k = k0 + c * E;
    const bool sum_bias = d.d_bias && k0 == 0;
    auto ask = [&](long long p0) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const long long p = p0 + row + u * kDown;
            const bool in = p < end;
            dy[u] = load_chunk((const T*)d.dy + p * d.ys + n, in ? d.N - n : 0);
            if (ACT != LP_ACT_NONE) pre[u] = load_chunk((const T*)d.pre + p * d.N + n, in ? d.N - n : 0);
            x[u] = load_chunk((const T*)d.x + p * d.xs + k, in ? d.K - k : 0);
        }
    };
    auto put = [&](int buffer) {
        char* to = lds + buffer * kStage;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int at = (row + u * kDown) * kPitch + c * 16;
            const Gradient<T> g = gradient<ACT>(dy[u], pre[u]);
            *(Chunk<T>*)(to + at) = g.hi;
            if (kSplit) *(Chunk<T>*)(to + 2 * kImage + at) = g.lo;
            *(Chunk<T>*)(to + kImage + at) = x[u];
#pragma unroll
            for (int j = 0; j < E; ++j) bias[j] += g.v[j];
        }
    };
    f32x16 acc[2][2] = {};
    if (first < end) {
        ask(first);
        put(0);
    }
    __syncthreads();
    int buffer = 0;
    for (long long p = first; p < end; p += kRows) {
        const bool more = p + kRows < end;
        if (more) ask(p + kRows);
        const char* from = lds + buffer * kStage;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int r = 0; r < kRows; r += 16) {
                Chunk<T> xv[2], g[2], lo[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    g[i] = columns<T>(from, r, wave_n + i * 32, lane);
                    if (kSplit) lo[i] = columns<T>(from + 2 * kImage, r, wave_n + i * 32, lane);
                    xv[i] = columns<T>(from + kImage, r, wave_k + i * 32, lane);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (kSplit) acc[i][j] = multiply(lo[i], xv[j], acc[i][j]);
                        acc[i][j] = multiply(g[i], xv[j], acc[i][j]);
                    }
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRows; r += 2) {
                float xv[2], g[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    g[i] = *(const float*)(from + (r + h) * kPitch + (wave_n + i * 32 + l32) * 4);
                    xv[i] = *(const float*)(from + kImage + (r + h) * kPitch + (wave_k + i * 32 + l32) * 4);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(g[i], xv[j], acc[i][j], 0, 0, 0);
            }
        }
        if (more) put(buffer ^ 1);
        __syncthreads();
        buffer ^= 1;
    }
    if (d.d_weight) {
        float* out = d.parts ? d.parts + (long long)split * d.N * d.K : d.d_weight;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int kk = k0 + wave_k + j * 32 + l32;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int nn = n0 + wave_n + i * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
                    if (kk >= d.K || nn >= d.N) continue;
                    float* at = out + (long long)nn * d.K + kk;
                    *at = d.parts ? acc[i][j][e] : *at + acc[i][j][e];
                }
            }
    }
    if (sum_bias) {
        float* sums = (float*)lds;   // [kDown][128]
#pragma unroll
        for (int j = 0; j < E; ++j) sums[row * kWeightTile + c * E + j] = bias[j];
        __syncthreads();
        if (threadIdx.x < kWeightTile && n0 + (int)threadIdx.x < d.N) {
            float sum = 0.0f;
            for (int r = 0; r < kDown; ++r) sum += sums[r * kWeightTile + threadIdx.x];
            const int nn = n0 + threadIdx.x;
            if (d.parts) d.bias_parts[(long long)split * d.N + nn] = sum;
            else d.d_bias[nn] += sum;
        }
    }
}

// out += the sum of its parts, in their order.
__global__ __launch_bounds__(kThreads) void linear_join_kernel(const float* parts, float* out, const float* bias_parts, float* d_bias, long long count, int N, int splits)
{
    const long long blocks = (count + kThreads - 1) / kThreads, all = blocks + (d_bias ? (N + kThreads - 1) / kThreads : 0);
    for (long long b = blockIdx.x; b < all; b += gridDim.x) {
        const bool weight = b < blocks;
        const long long i = (weight ? b : b - blocks) * kThreads + threadIdx.x, size = weight ? count : N;
        const float* from = weight ? parts : bias_parts;
        float* to = weight ? out : d_bias;
        if (!to || i >= size) continue;
        float sum = 0.0f;
        for (int s = 0; s < splits; ++s) sum += from[s * size + i];
        to[i] += sum;
    }
}

// W^T with rows of `pitch` elements.
template <class T>
__global__ __launch_bounds__(kThreads) void linear_turn_kernel(const T* w, int N, int K, T* out, long long pitch)
{
    __shared__ T tile[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const long long blocks_k = (K + 31) / 32, blocks = blocks_k * ((N + 31) / 32);
    for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int k0 = (int)(b % blocks_k) * 32, n0 = (int)(b / blocks_k) * 32;
        __syncthreads();
        for (int r = y; r < 32; r += 8)
            if (n0 + r < N && k0 + x < K) tile[r][x] = w[(long long)(n0 + r) * K + k0 + x];
        __syncthreads();
        for (int r = y; r < 32; r += 8)
            if (k0 + r < K && n0 + x < N) out[(k0 + r) * pitch + n0 + x] = tile[x][r];
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int dtype_bytes(int t) { return t == LP_F32 ? 4 : 2; }

struct Call {
    long long P, xs, ys, rs;
    int K, N, act, dtype;
    const void *weight, *residual;
    const float* bias;
};

lp_status validate(const lp_linear* q, Call* c)
{
    if (!q) return fail(LP_ERR_INVALID_ARG, "linear must not be NULL");
    if (q->P < 0) return fail(LP_ERR_INVALID_ARG, "linear->P must be >= 0");
    if (q->K < 1 || q->N < 1) return fail(LP_ERR_INVALID_ARG, "linear->K and linear->N must be >= 1");
    if (q->K > 1 << 20 || q->N > 1 << 20) return fail(LP_ERR_UNSUPPORTED, "linear->K and linear->N are at most 2^20");
    if (q->act < LP_ACT_NONE || q->act > LP_ACT_GELU) return fail(LP_ERR_INVALID_ARG, "linear->act must be an lp_act");
    if (q->dtype != LP_F32 && q->dtype != LP_BF16 && q->dtype != LP_F16)
        return fail(LP_ERR_INVALID_ARG, "linear->dtype must be LP_F32, LP_BF16 or LP_F16");
    c->P = q->P; c->K = q->K; c->N = q->N; c->act = q->act; c->dtype = q->dtype;
    c->xs = q->x_stride ? q->x_stride : q->K;
    c->ys = q->y_stride ? q->y_stride : q->N;
    c->rs = q->r_stride ? q->r_stride : q->N;
    if (c->xs < q->K || c->ys < q->N || c->rs < q->N)
        return fail(LP_ERR_INVALID_ARG, "linear's strides must be 0 or at least the number of channels");
    const double most = (double)q->P * std::fmax((double)c->xs, std::fmax((double)c->ys, (double)c->rs)) * 4.0;
    if (most > 4e18) return fail(LP_ERR_UNSUPPORTED, "linear: tensors beyond 64-bit offsets");
    c->weight = q->weight; c->residual = q->residual; c->bias = q->bias;
    return LP_OK;
}

// How the positions are divided for the parameters' gradients.
struct Parts {
    int tiles_n, tiles_k, splits;
    long long chunk;
};
Parts parts_of(const Call& c, int n_cu)
{
    Parts p;
    p.tiles_n = (c.N + kWeightTile - 1) / kWeightTile;
    p.tiles_k = (c.K + kWeightTile - 1) / kWeightTile;
    const long long tiles = (long long)p.tiles_n * p.tiles_k, target = (2ll * n_cu + tiles - 1) / tiles, most = (c.P + 255) / 256;
    long long splits = target < most ? target : most;
    if (splits < 1) splits = 1;
    p.chunk = ((c.P + splits - 1) / splits + 31) / 32 * 32;
    if (p.chunk < 32) p.chunk = 32;
    p.splits = (int)((c.P + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    return p;
}

struct Sizes {
    size_t turned, parts, bias_parts;
};
Sizes sizes(const Call& c, int n_cu)
{
    const Parts p = parts_of(c, n_cu);
    const size_t E = 16 / dtype_bytes(c.dtype);
    Sizes s;
    s.turned = align256((size_t)c.K * ((c.N + E - 1) / E * E) * dtype_bytes(c.dtype));
    s.parts = p.splits > 1 ? align256((size_t)p.splits * c.N * c.K * sizeof(float)) : 0;
    s.bias_parts = p.splits > 1 ? align256((size_t)p.splits * c.N * sizeof(float)) : 0;
    return s;
}

template <class T> struct Type { using type = T; };
// Calls f with the type and the activation as constants.
template <class F>
void dispatch(int dtype, int act, F&& f)
{
    auto typed = [&](auto t) {
        switch (act) {
            case LP_ACT_RELU: f(t, std::integral_constant<int, LP_ACT_RELU>()); break;
            case LP_ACT_SILU: f(t, std::integral_constant<int, LP_ACT_SILU>()); break;
            case LP_ACT_GELU: f(t, std::integral_constant<int, LP_ACT_GELU>()); break;
            default: f(t, std::integral_constant<int, LP_ACT_NONE>());
        }
    };
    if (dtype == LP_BF16) typed(Type<__bf16>());
    else if (dtype == LP_F16) typed(Type<_Float16>());
    else typed(Type<float>());
}

unsigned grid_of(long long n) { return (unsigned)(n < kMaxGrid ? n : kMaxGrid); }

lp_status launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LP_OK : fail(LP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

lp_status aligned(int dtype, std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if ((uintptr_t)p % dtype_bytes(dtype)) return fail(LP_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    return LP_OK;
}

// Tiles of 128 x 128 results, narrower ones where there are few channels.
template <class T, int ACT, bool BACK>
void tiles(LinearDev d, hipStream_t s)
{
    auto go = [&](auto bn) {
        constexpr int BN = decltype(bn)::value;
        d.tiles_p = (d.P + 127) / 128;
        d.tiles_n = (d.N + BN - 1) / BN;
        const long long tiles = d.tiles_p * d.tiles_n;
        hipLaunchKernelGGL((linear_tile_kernel<T, ACT, BACK, 128, BN>), dim3(grid_of((tiles + 7) / 8 * 8)), dim3(kThreads), 0, s, d);
    };
    if (d.N <= 32) go(std::integral_constant<int, 32>());
    else if (d.N <= 64) go(std::integral_constant<int, 64>());
    else go(std::integral_constant<int, 128>());
}

lp_status forward(const lp_linear* q, const void* x, void* y, void* pre, void* workspace, size_t workspace_bytes, hipStream_t s)
{
    Call c;
    lp_status st = validate(q, &c);
    if (st != LP_OK) return st;
    if (c.P == 0) return LP_OK;
    if (!x || !y || !c.weight) return fail(LP_ERR_INVALID_ARG, "x, y and linear->weight must not be NULL");
    if ((st = aligned(c.dtype, {x, y, pre, c.weight, c.residual})) != LP_OK) return st;
    (void)workspace;
    (void)workspace_bytes;
    LinearDev d;
    std::memset(&d, 0, sizeof(d));
    d.P = c.P; d.K = c.K; d.N = c.N; d.as = c.xs; d.ys = c.ys; d.rs = c.rs;
    d.a = x; d.w = c.weight; d.ws = c.K; d.res = c.residual; d.bias = c.bias; d.out = y; d.keep = pre;
    dispatch(c.dtype, c.act, [&](auto t, auto act) {
        using T = typename decltype(t)::type;
        constexpr int A = decltype(act)::value;
        const dim3 rows_grid((c.N + kThreads / 64 * kOutputs - 1) / (kThreads / 64 * kOutputs));
        if (c.P == 1) hipLaunchKernelGGL((linear_rows_kernel<T, A, 1>), rows_grid, dim3(kThreads), 0, s, d);
        else if (c.P <= 4) hipLaunchKernelGGL((linear_rows_kernel<T, A, 4>), rows_grid, dim3(kThreads), 0, s, d);
        else if (c.P <= kFewRows) hipLaunchKernelGGL((linear_rows_kernel<T, A, kFewRows>), rows_grid, dim3(kThreads), 0, s, d);
        else tiles<T, A, false>(d, s);
    });
    return launched("linear forward launch");
}

lp_status backward(const lp_linear* q, const void* x, const void* pre, const void* d_y, void* d_x, float* d_weight, float* d_bias,
                   void* workspace, size_t workspace_bytes, hipStream_t s)
{
    Call c;
    lp_status st = validate(q, &c);
    if (st != LP_OK) return st;
    if (c.P == 0) return LP_OK;
    if (!d_y || (d_weight && !x) || (d_x && !c.weight)) return fail(LP_ERR_INVALID_ARG, "d_y, x and linear->weight must not be NULL");
    if (c.act != LP_ACT_NONE && !pre) return fail(LP_ERR_INVALID_ARG, "pre must not be NULL with an activation");
    if ((st = aligned(c.dtype, {x, pre, d_y, d_x, c.weight})) != LP_OK) return st;
    std::string err;
    int n_cu = 0;
    if (compute_units(&n_cu, &err)) return fail(LP_ERR_HIP, err);
    const Sizes size = sizes(c, n_cu);
    if (!workspace || workspace_bytes < size.turned + size.parts + size.bias_parts)
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_linear_workspace_bytes");
    if ((uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const Parts p = parts_of(c, n_cu);
    char* at = (char*)workspace;
    dispatch(c.dtype, c.act, [&](auto t, auto act) {
        using T = typename decltype(t)::type;
        constexpr int A = decltype(act)::value;
        if (d_x) {
            const long long pitch = (c.N + kChunk<T> - 1) / kChunk<T> * kChunk<T>;
            const long long blocks = ((c.K + 31ll) / 32) * ((c.N + 31ll) / 32);
            hipLaunchKernelGGL((linear_turn_kernel<T>), dim3(grid_of(blocks)), dim3(kThreads), 0, s, (const T*)c.weight, c.N, c.K, (T*)at, pitch);
            LinearDev d;
            std::memset(&d, 0, sizeof(d));
            d.P = c.P; d.K = c.N; d.N = c.K; d.as = c.ys; d.ys = c.xs;
            d.a = d_y; d.pre = pre; d.w = at; d.ws = pitch; d.out = d_x;
            tiles<T, A, true>(d, s);
        }
        if (d_weight || d_bias) {
            WeightDev d;
            std::memset(&d, 0, sizeof(d));
            d.P = c.P; d.K = d_weight ? c.K : 0; d.N = c.N; d.xs = c.xs; d.ys = c.ys;
            d.x = x; d.dy = d_y; d.pre = pre; d.d_weight = d_weight; d.d_bias = d_bias;
            d.parts = p.splits > 1 ? (float*)(at + size.turned) : nullptr;
            d.bias_parts = p.splits > 1 ? (float*)(at + size.turned + size.parts) : nullptr;
            d.chunk = p.chunk; d.tiles_n = p.tiles_n; d.tiles_k = d_weight ? p.tiles_k : 1; d.splits = p.splits;
            hipLaunchKernelGGL((linear_weight_kernel<T, A>), dim3((unsigned)(d.tiles_n * d.tiles_k * p.splits)), dim3(kThreads), 0, s, d);
            if (p.splits > 1) {
                const long long count = d_weight ? (long long)c.N * c.K : 0;
                const long long blocks = (count + kThreads - 1) / kThreads + (c.N + kThreads - 1) / kThreads;
                hipLaunchKernelGGL(linear_join_kernel, dim3(grid_of(blocks)), dim3(kThreads), 0, s, d.parts, d_weight, d.bias_parts, d_bias, count, c.N, p.splits);
            }
        }
    });
    return launched("linear backward launch");
}

}  // namespace

}  // namespace lp

extern "C" {

lp_status lp_linear_workspace_bytes(const lp_linear* linear, size_t* fwd_bytes, size_t* bwd_bytes)
try {
    lp::Call c;
    const lp_status st = lp::validate(linear, &c);
    if (st != LP_OK) return st;
    if (fwd_bytes) *fwd_bytes = 0;
    if (!bwd_bytes) return LP_OK;
    std::string err;
    int n_cu = 0;
    if (lp::compute_units(&n_cu, &err)) return lp::fail(LP_ERR_HIP, err);
    const lp::Sizes size = lp::sizes(c, n_cu);
    *bwd_bytes = size.turned + size.parts + size.bias_parts;
    return LP_OK;
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_linear_fwd(const lp_linear* linear, const void* x, void* y, void* pre, void* workspace, size_t workspace_bytes, void* stream)
try {
    return lp::forward(linear, x, y, pre, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_linear_bwd(const lp_linear* linear, const void* x, const void* pre, const void* d_y, void* d_x, float* d_weight,
                        float* d_bias, void* workspace, size_t workspace_bytes, void* stream)
try {
    return lp::backward(linear, x, pre, d_y, d_x, d_weight, d_bias, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

}  // extern "C"
