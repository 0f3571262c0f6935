// Device code and declarations that the translation units of the products with a weight matrix share (lp_linear*.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lp_act.h"
#include "lp_kernels.h"

namespace lp {
namespace linear {

using namespace act;

constexpr int kThreads = 256;
constexpr unsigned kMaxGrid = 1u << 30;
// Where a call moves more than the Infinity Cache holds, results are stored past the caches: they would only drive out what is yet to
// be read (65536 x 512 -> 2048 in bf16 with pre, 0.6 GB: 272 -> 238 us in the tile loop of that time; 160^3 x 32 -> 64 in fp32, whose x no other
// workgroup reads, takes the same either way).
constexpr double kCacheBytes = 256e6;
inline unsigned grid_of(long long n) { return (unsigned)(n < kMaxGrid ? n : kMaxGrid); }

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
// WHOLE: rows end with whole chunks.  Else all lanes that reach behind a row's end do so by as much (it is the end of the same row size):
// what is left is moved in pieces of 8, 4 and 2 bytes, whose sizes are the same for all of them.
template <bool WHOLE, class T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, long long count)
{
    u32x4 w = {0, 0, 0, 0};
    if (count >= (WHOLE ? 1 : kChunk<T>)) {
        __builtin_memcpy(&w, p, 16);
    } else if (!WHOLE && count > 0) {
        const char* at = (const char*)p;
        const int bytes = __builtin_amdgcn_readfirstlane((int)count) * (int)sizeof(T);
        if (bytes & 8) {
            u32x2 v;
            __builtin_memcpy(&v, at, 8);
            w[0] = v[0];
            w[1] = v[1];
        }
        if (bytes & 4) {
            uint32_t v;
            __builtin_memcpy(&v, at + (bytes & 8), 4);
            if (bytes & 8) w[2] = v; else w[0] = v;
        }
        if (sizeof(T) == 2 && bytes & 2) {
            uint16_t v;
            __builtin_memcpy(&v, at + (bytes & 12), 2);
            switch (bytes & 12) {
                case 0: w[0] = v; break;
                case 4: w[1] = v; break;
                case 8: w[2] = v; break;
                default: w[3] = v;
            }
        }
    }
    return __builtin_bit_cast(Chunk<T>, w);
}
// past_cache: see kCacheBytes.
template <bool WHOLE, class T>
__device__ __forceinline__ void store_chunk(T* p, long long count, const Chunk<T>& c, bool past_cache = false)
{
    const u32x4 w = __builtin_bit_cast(u32x4, c);
    if (count >= (WHOLE ? 1 : kChunk<T>)) {
        if (past_cache) {
            typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(2)));
            asm volatile("" ::: "memory");   // (with nothing around it both stores would become one ordinary one)
            __builtin_nontemporal_store((Any)w, (Any*)p);
            asm volatile("" ::: "memory");
        } else {
            __builtin_memcpy(p, &w, 16);
        }
    } else if (!WHOLE && count > 0) {
        char* at = (char*)p;
        const int bytes = __builtin_amdgcn_readfirstlane((int)count) * (int)sizeof(T);
        if (bytes & 8) {
            const u32x2 v = {w[0], w[1]};
            __builtin_memcpy(at, &v, 8);
        }
        if (bytes & 4) {
            const uint32_t v = bytes & 8 ? w[2] : w[0];
            __builtin_memcpy(at + (bytes & 8), &v, 4);
        }
        if (sizeof(T) == 2 && bytes & 2) {
            const uint16_t v = (uint16_t)((bytes & 12) == 0 ? w[0] : (bytes & 12) == 4 ? w[1] : (bytes & 12) == 8 ? w[2] : w[3]);
            __builtin_memcpy(at + (bytes & 12), &v, 2);
        }
    }
}

// acc += a b^T over the channels of two neighbouring chunks of a row, of which lanes 0 .. 31 hold the first, lanes 32 .. 63 the second
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

// The GELU and its slope for tensors of 16 bits, whose results are rounded by 2^-12 and more (a slope's product with d_y by 2^-16 in two
// parts).  As in lp_act.h the tail of the normal distribution beyond |z| is t Q(t) exp(-z^2 / 2), t = 1 / (1 + p |z|), but
// with one Q of degree 4 for all z: for the value a fit of least relative error of the tail (3.6e-5 with fp32 rounding, so a negative z's value
// stays within a seventh of half a step of fp16), for the slope one of least absolute error (3.1e-7).  20 instructions' time instead of
// 31: the vector instructions of the activation bound wide blocks as much as the matrix cores.
__device__ __forceinline__ float tail_of(float z, float& e, float p, const float (&q)[5])
{
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    const float t = __builtin_amdgcn_rcpf(fmaf(p, fabsf(z), 1.0f));
    float v = q[4];
#pragma unroll
    for (int k = 3; k >= 0; --k) v = fmaf(v, t, q[k]);
    return v * t * e;
}
template <int ACT, class T>
__device__ __forceinline__ float activate_as(float z)
{
    if constexpr (ACT == LP_ACT_GELU && sizeof(T) == 2) {
        float e;
        const float tail = tail_of(z, e, 0.38f, {0.151225137f, 0.157829468f, 0.0919797578f, 0.188876449f, -0.08992834f});
        return fmaf(-fminf(fabsf(z), 64.0f), tail, fmaxf(z, 0.0f));   // (of an infinite z the tail is 0, and of NaN it is NaN)
    } else {
        return activate<ACT>(z);
    }
}
template <int ACT, class T>
__device__ __forceinline__ float slope_as(float z)
{
    if constexpr (ACT == LP_ACT_GELU && sizeof(T) == 2) {
        float e;
        const float tail = tail_of(z, e, 0.34f, {0.130569511f, 0.179848642f, -0.0278562922f, 0.320559185f, -0.103121231f});
        return fmaf(z * kInvSqrt2Pi, e, 0.5f + __builtin_copysignf(0.5f - tail, z));
    } else {
        return slope<ACT>(z);
    }
}

// d_z of a chunk, rounded to T, what that left, rounded to T (of fp16: to bf16, and there is no third part), and what that left.
template <class T>
struct Gradient {
    Chunk<T> part[3];
    float v[kChunk<T>];
};
template <int ACT, class T>
__device__ __forceinline__ Gradient<T> gradient(const Chunk<T>& dy, const Chunk<T>& pre)
{
    Gradient<T> g;
#pragma unroll
    for (int j = 0; j < kChunk<T>; ++j) {
        g.v[j] = (float)dy.v[j] * (ACT == LP_ACT_NONE ? 1.0f : slope_as<ACT, T>((float)pre.v[j]));
        float rest = g.v[j];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            asm("" : "+v"(rest));   // (a part and what it leaves come from one value: the first could be rounded straight from the product)
            if (k == 0) g.v[j] = rest;
            if constexpr (std::is_same<T, _Float16>::value) {
                if (k == 1) {
                    g.part[k].v[j] = __builtin_bit_cast(_Float16, (__bf16)rest);
                    break;
                }
            }
            g.part[k].v[j] = (T)rest;
            rest -= (float)g.part[k].v[j];   // (an infinite d_z leaves NaN)
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
    int past_cache;                 // results are stored past the caches
    float* parts;                   // of the general kernel: sums of a part of the steps
    int splits, split_steps;        // parts, steps of one
};

// Where a chunk of a row of 128 bytes lies in LDS.  Two neighbouring rows fill the 64 banks once; turned over by row / 2, the same chunk of 16
// neighbouring rows, which a matrix operand reads at once, touches every bank once too, and so do a row pair's chunks, which are written at once.
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * 128 + ((chunk ^ (row >> 1 & 7)) << 4); }

// Tile of a workgroup: neighbouring workgroups go to the chip's eight XCDs in turn, so each of these takes one run of the
// tiles; channels' tiles of the same positions follow one another (their positions are read from the XCD's L2).
__device__ __forceinline__ long long tile_of(long long b, long long tiles)
{
    const long long each = (tiles + 7) / 8;
    return (b & 7) * each + (b >> 3);
}

__device__ __forceinline__ u32x2 read_transposed(const char* at)
{
    typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4 Lds;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)at));
}

// The results of a wave's blocks of 32 x 32 (channels, positions) for positions p0 .. and channels n0 ..: value e of a lane is channel
// 8 (e / 4) + 4 h + e % 4 of position l32 of a block.  They are turned over in the wave's own LDS, 32 positions at a time, so that
// neighbouring lanes write neighbouring channels.
// The residual of 32 positions (of the lane's chunks) may have been asked for before.
template <class T, int BLOCKS_N> constexpr int kFinishTimes = 32 / (64 / (32 * BLOCKS_N / kChunk<T>));   // chunks of a lane
template <class T, bool WHOLE, int BLOCKS_N>
__device__ __forceinline__ void ask_residual(const LinearDev& d, long long p0, int n0, int lane, Chunk<T> (&added)[kFinishTimes<T, BLOCKS_N>])
{
    constexpr int kAcross = 32 * BLOCKS_N / kChunk<T>, kDown = 64 / kAcross;
    const int n = n0 + lane % kAcross * kChunk<T>;
    const long long first = p0 + lane / kAcross;
    const T* res = (const T*)d.res + first * d.rs + n;
#pragma unroll
    for (int r = 0; r < kFinishTimes<T, BLOCKS_N>; ++r)
        added[r] = load_chunk<WHOLE>(res + r * kDown * d.rs, first + r * kDown < d.P ? d.N - n : 0);
}
template <class T, int ACT, bool BACK, bool WHOLE, int BLOCKS_P, int BLOCKS_N>
__device__ __forceinline__ void finish(const LinearDev& d, const f32x16 (&acc)[BLOCKS_N][BLOCKS_P], float* turn, long long p0, int n0, int lane,
                                       const Chunk<T> (*asked)[kFinishTimes<T, BLOCKS_N>] = nullptr)
{
    constexpr int E = kChunk<T>, kAcross = 32 * BLOCKS_N / E, kDown = 64 / kAcross, kPitch = 32 * BLOCKS_N + 4;
    constexpr int kTimes = kFinishTimes<T, BLOCKS_N>;
    const int l32 = lane & 31, h = lane >> 5, n = n0 + lane % kAcross * E;
    const long long first = p0 + lane / kAcross;   // the lane's first position; the others follow at distances that all lanes share
    float bias[E];
#pragma unroll
    for (int j = 0; j < E; ++j) bias[j] = d.bias && n + j < d.N ? d.bias[n + j] : 0.0f;
    T *out = (T*)d.out + first * d.ys + n, *keep = (T*)d.keep + first * d.N + n;
#pragma unroll
    for (int jp = 0; jp < BLOCKS_P; ++jp) {
#pragma unroll
        for (int i = 0; i < BLOCKS_N; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *(f32x4*)(turn + l32 * kPitch + i * 32 + 2 * e + 4 * h) = f32x4{acc[i][jp][e], acc[i][jp][e + 1], acc[i][jp][e + 2], acc[i][jp][e + 3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        int count[kTimes];
        Chunk<T> added[kTimes];
#pragma unroll
        for (int r = 0; r < kTimes; ++r) {
            count[r] = first + (jp * 32 + r * kDown) < d.P ? d.N - n : 0;
            added[r] = Chunk<T>{};
        }
        if (!BACK && d.res) {
            if (asked) {
#pragma unroll
                for (int r = 0; r < kTimes; ++r) added[r] = (*asked)[r];
            } else {
                ask_residual<T, WHOLE, BLOCKS_N>(d, p0 + jp * 32, n0, lane, added);
            }
        }
        // (whether there is a residual stands outside the loop: 1 to 2 % of a call without one)
        auto store_all = [&](auto residual) {
#pragma unroll
            for (int r = 0; r < kTimes; ++r) {
                float z[E];
                const float* from = turn + (r * kDown + lane / kAcross) * kPitch + lane % kAcross * E;
#pragma unroll
                for (int j = 0; j < E; j += 4) *(f32x4*)(z + j) = *(const f32x4*)(from + j);
                Chunk<T> v;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    z[j] += bias[j];
                    v.v[j] = (T)z[j];
                }
                if (!BACK) {
                    if (d.keep) store_chunk<WHOLE>(keep + (long long)(jp * 32 + r * kDown) * d.N, count[r], v, d.past_cache);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float y = activate_as<ACT, T>(z[j]);
                        v.v[j] = (T)(decltype(residual)::value ? y + (float)added[r].v[j] : y);
                    }
                }
                store_chunk<WHOLE>(out + (jp * 32 + r * kDown) * d.ys, count[r], v, d.past_cache);
            }
        };
        if (!BACK && d.res) store_all(std::true_type());
        else store_all(std::false_type());
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- launchers -------------------------------------------------------------------------------------------------

// Calls f with the activation as a constant.
template <class F>
void with_act_of(int act, F&& f)
{
    switch (act) {
        case LP_ACT_RELU: f(std::integral_constant<int, LP_ACT_RELU>()); break;
        case LP_ACT_SILU: f(std::integral_constant<int, LP_ACT_SILU>()); break;
        case LP_ACT_GELU: f(std::integral_constant<int, LP_ACT_GELU>()); break;
        default: f(std::integral_constant<int, LP_ACT_NONE>());
    }
}

// Whether rows end with whole chunks.
inline bool whole(const LinearDev& d, int dtype) { return d.K % (dtype == LP_F32 ? 4 : 8) == 0 && d.N % (dtype == LP_F32 ? 4 : 8) == 0; }

// The general kernel (lp_linear_tile.hip).  back: d_x from d_y and pre.  d.splits > 1: with d.parts.
constexpr int kTileP = 128;
inline int tile_channels(int made) { return made <= 32 ? 32 : made <= 64 ? 64 : 128; }
void launch_tiles(int dtype, int act, bool back, LinearDev d, hipStream_t s);

// Few channels (lp_linear_stream.hip).  back: d_x from d_y and pre, fp32 alone; the weight is W as it is, with rows of ws elements.
inline bool is_few(int dtype, int summed, int made) { return made <= 128 && summed * (dtype == LP_F32 ? 4 : 2) <= 256; }
void launch_stream(int dtype, int act, bool back, const LinearDev& d, int n_cu, hipStream_t s);

// 16-bit types, more than 128 channels (lp_linear_wide.hip): the weights in the operands' order, and the products with them.
__host__ __device__ constexpr int wide_blocks(int k) { return (k + 63) / 64 * 4; }   // of 16 summed channels
void launch_pack(int dtype, bool turned, const void* w, int rows, int cols, int pitch, void* out, hipStream_t s);
void launch_wide(int dtype, int act, bool back, LinearDev d, hipStream_t s);   // back: act is LP_ACT_NONE

// 16-bit types, gradients of the parameters, and d_x where there are few channels (lp_linear_back_*.hip; whole: rows end with whole chunks).
struct BackDev {
    long long P;
    int K, N;
    int x_channels;              // of x that are read: K, or 0 where d_weight is not wanted (x may be NULL then)
    long long xs, ys;
    const void *x, *dy, *pre, *w;
    void *d_x, *dz;              // dz: [P][N]
    float *parts, *bias_parts;   // [splits][N][K], [splits][N]
    long long chunk;             // positions of a part
    int tiles_n, tiles_k, splits;
    int d_weight, d_bias;        // wanted
};

// How the positions are divided for the parameters' gradients.
struct Parts {
    int bn, bk, tiles_n, tiles_k, splits;
    long long chunk;
};
hipError_t launch_back_bf16_whole(int act, const BackDev& d, const Parts& p, bool skinny, hipStream_t s);
hipError_t launch_back_bf16_any(int act, const BackDev& d, const Parts& p, bool skinny, hipStream_t s);
hipError_t launch_back_f16_whole(int act, const BackDev& d, const Parts& p, bool skinny, hipStream_t s);
hipError_t launch_back_f16_any(int act, const BackDev& d, const Parts& p, bool skinny, hipStream_t s);

}  // namespace linear
}  // namespace lp
