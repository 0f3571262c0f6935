// The gradients' kernel of 16-bit types, for the translation units of each type and of rows that end with whole chunks or not.
#pragma once
#include "lp_linear.h"

namespace lp {
namespace linear {

namespace {

// ---- gradients in 16-bit types ---------------------------------------------------------------------------------
//
// A workgroup takes a part of the positions, some at a time: d_z is made from d_y and pre in registers, split in parts and
// laid into LDS beside x, and from there come all products of these positions: d_z^T x in 32 x 32 blocks, and, where all channels of d_z are there
// (SKINNY: up to 128 -> 128 channels), d_z W too, in 16 x 16 blocks with W^T as operands in LDS.  Then everything is read once and d_x is written once.
// Blocks with more channels: workgroups of 128 channels of d_z x up to 512 of x, so that d_z is made once for 512 channels of x; the first of
// them writes d_z rounded to 16 bits for the product with W, which another kernel makes.  There one workgroup fills a compute unit; of two
// waves that share a SIMD one multiplies first and then makes the next positions' d_z, the other one the other way round, so that the
// vector instructions of one run under the matrix instructions of the other.
//
// Measured with GELU in bf16, all gradients: 24 x 256^2 positions, 32 -> 128 channels 278 to 300 us for 1.0 GB, 65536 x 512 -> 2048 590 us, of which this
// kernel takes 412 (0.41 TFLOP for d_W's three parts: 1.0 PFLOP/s).
// Parts of d_z.  The sums' own error goes by the length of a part of the positions, not by their number, and stays below 1.4e-6 (64 -> 64 channels,
// 1.6 million positions; up to 65536 positions 3e-7 to 8e-7): in bf16 two parts, 17 bits, would leave 2.5e-6 at every size, so there are three, whatever the number of
// positions.  What that costs, against two: 512 -> 2048 channels, 16384 positions 195 and 174 us, 65536 590 and 510, 262144 2215 and 1890; 32 -> 128,
// 262144 positions 65 and 56, 1.6 million 300 and 262.  (d_W against 64 bits at 65536 x 512 -> 2048: 8e-7, with two 2.5e-6.)  Of fp16 two parts
// have 19 bits: 5e-7.
// d_z W takes the first part alone: d_x, itself rounded to 16 bits, is 2.3e-3 off in bf16 then and 1.7e-3 with all of d_z.  A second part would double
// that product (150 of the 590 us above) and, beyond 128 channels, the 0.5 GB that are written and read of d_z.

__host__ __device__ constexpr int image_pitch(int channels) { return channels * 2 + (channels * 2 % 256 == 64 ? 0 : 64); }

template <int BN, int BK, int WN, int WK, int ROWS, bool SKINNY>
struct BackShape {
    static constexpr int kBN = BN, kBK = BK, kWN = WN, kWK = WK, kRows = ROWS;
    static constexpr bool kSkinny = SKINNY;
    static constexpr int kWaves = SKINNY ? 4 : WN * WK, kThreadsOf = 64 * kWaves;
    static constexpr int kPitchN = image_pitch(BN), kPitchK = image_pitch(BK);
    static constexpr int kBlocksN = BN / WN / 32, kBlocksK = BK / WK / 32;
    static constexpr int kLoadsN = ROWS * (BN / 8) / kThreadsOf, kLoadsK = ROWS * (BK / 8) / kThreadsOf;
    static_assert(ROWS * (BN / 8) % kThreadsOf == 0 && ROWS * (BK / 8) % kThreadsOf == 0);
    static constexpr int kImageN = ROWS * kPitchN, kImageK = ROWS * kPitchK;
    static constexpr int kWeights = SKINNY ? BN * BK * 2 : 0;
    static constexpr int stage(int parts) { return kImageN * parts + kImageK; }
    static constexpr int lds(int parts) { return stage(parts) * (SKINNY ? 1 : 2) + kWeights; }
};

template <class T, int PITCH>
__device__ __forceinline__ Chunk<T> operand(const char* image, int r0, int column, int lane)
{
    const int q = lane >> 4, t = lane & 15;
    const char* at = image + (r0 + 4 * (q >> 1) + (t >> 2)) * PITCH + (column + 16 * (q & 1) + 4 * (t & 3)) * 2;
    const u32x2 a = read_transposed(at), b = read_transposed(at + 8 * PITCH);
    return __builtin_bit_cast(Chunk<T>, u32x4{a[0], a[1], b[0], b[1]});
}
__device__ __forceinline__ f32x4 multiply16(const Chunk<__bf16>& a, const Chunk<__bf16>& b, f32x4 acc)
{
    using V = Vec<__bf16>::Of;
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply16(const Chunk<_Float16>& a, const Chunk<_Float16>& b, f32x4 acc)
{
    using V = Vec<_Float16>::Of;
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
}

// PARTS: 16-bit parts of d_z.
template <class T, int ACT, int PARTS, bool WHOLE, class S>
__global__ __launch_bounds__(S::kThreadsOf, S::kSkinny && (S::kBN < 128 || S::kBK < 128) ? 3 : 2) void linear_back_kernel(BackDev d)
{
    constexpr bool kSlope = ACT != LP_ACT_NONE;
    constexpr int kStage = S::stage(PARTS), kX = S::kImageN * PARTS;
    constexpr int kAcrossN = S::kBN / 8, kDownN = S::kThreadsOf / kAcrossN, kAcrossK = S::kBK / 8, kDownK = S::kThreadsOf / kAcrossK;
    extern __shared__ char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
    const int cn = threadIdx.x % kAcrossN, rn = threadIdx.x / kAcrossN, ck = threadIdx.x % kAcrossK, rk = threadIdx.x / kAcrossK;
    const bool multiplies = wave < S::kWN * S::kWK && d.d_weight;
    const int wave_n = wave / S::kWK * (S::kBlocksN * 32), wave_k = wave % S::kWK * (S::kBlocksK * 32);
    const int tiles = d.tiles_n * d.tiles_k, split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int n0 = tile / d.tiles_k * S::kBN, k0 = tile % d.tiles_k * S::kBK;
    const long long first = split * d.chunk, end = min(d.P, first + d.chunk);
    const int n = n0 + cn * 8, k = k0 + ck * 8;
    const bool write_dz = d.dz && k0 == 0;
    Chunk<T> dy[S::kLoadsN], pre[S::kLoadsN], x[S::kLoadsK];
    float bias[8] = {};
    // A row's last chunk, where it is not whole, is read as the row's last 16 bytes and shifted when it is used: piece by piece the loads
    // would be waited for one after the other (131979 x 72 -> 97 in fp16: 85 us instead of 65).  (Rows of less than a chunk are.)
    const bool long_n = WHOLE || d.N >= 8, long_k = WHOLE || d.K >= 8;
    const int shift_n = !WHOLE && long_n && n < d.N && n + 8 > d.N ? n + 8 - d.N : 0, shift_k = !WHOLE && long_k && k < d.K && k + 8 > d.K ? k + 8 - d.K : 0;
    // a lane's rows of the next positions; those of its other loads lie at distances that all lanes share
    const T *dy_at = (const T*)d.dy + (first + rn) * d.ys + n - shift_n, *pre_at = (const T*)d.pre + (first + rn) * d.N + n - shift_n,
            *x_at = (const T*)d.x + (first + rk) * d.xs + k - shift_k;
    T* dz_at = (T*)d.dz + (first + rn) * d.N + n;
    auto ask = [&](long long p0) {
        const int left = (int)min((long long)S::kRows, end - p0);   // (<= 0 behind the last position)
        if (long_n) {
#pragma unroll
            for (int u = 0; u < S::kLoadsN; ++u) {
                const int in = rn + u * kDownN < left ? d.N - n : 0;
                dy[u] = load_chunk<true>(dy_at + u * kDownN * d.ys, in);
                if (kSlope) pre[u] = load_chunk<true>(pre_at + (long long)u * kDownN * d.N, in);
            }
        } else {
#pragma unroll
            for (int u = 0; u < S::kLoadsN; ++u) {
                const int in = rn + u * kDownN < left ? d.N - n : 0;
                dy[u] = load_chunk<false>(dy_at + u * kDownN * d.ys, in);
                if (kSlope) pre[u] = load_chunk<false>(pre_at + (long long)u * kDownN * d.N, in);
            }
        }
        if (long_k) {
#pragma unroll
            for (int u = 0; u < S::kLoadsK; ++u) x[u] = load_chunk<true>(x_at + u * kDownK * d.xs, rk + u * kDownK < left ? d.x_channels - k : 0);
        } else {
#pragma unroll
            for (int u = 0; u < S::kLoadsK; ++u) x[u] = load_chunk<false>(x_at + u * kDownK * d.xs, rk + u * kDownK < left ? d.x_channels - k : 0);
        }
        dy_at += S::kRows * d.ys;
        pre_at += (long long)S::kRows * d.N;
        x_at += S::kRows * d.xs;
    };
    auto shifted = [&](const Chunk<T>& c, int by) {
        return WHOLE ? c : __builtin_bit_cast(Chunk<T>, __builtin_bit_cast(unsigned __int128, c) >> (by * 16));
    };
    auto put = [&](char* to, long long p0) {
        const int left = (int)min((long long)S::kRows, end - p0);
#pragma unroll
        for (int u = 0; u < S::kLoadsN; ++u) {
            const int at = (rn + u * kDownN) * S::kPitchN + cn * 16;
            const Gradient<T> g = gradient<ACT>(shifted(dy[u], shift_n), shifted(pre[u], shift_n));
#pragma unroll
            for (int i = 0; i < PARTS; ++i) *(Chunk<T>*)(to + i * S::kImageN + at) = g.part[i];
#pragma unroll
            for (int j = 0; j < 8; ++j) bias[j] += g.v[j];
            if (write_dz) store_chunk<WHOLE>(dz_at + (long long)u * kDownN * d.N, rn + u * kDownN < left ? d.N - n : 0, g.part[0]);
        }
        dz_at += (long long)S::kRows * d.N;
#pragma unroll
        for (int u = 0; u < S::kLoadsK; ++u) *(Chunk<T>*)(to + kX + (rk + u * kDownK) * S::kPitchK + ck * 16) = shifted(x[u], shift_k);
    };
    f32x16 acc[S::kBlocksN][S::kBlocksK] = {};
    auto multiply_all = [&](const char* from) {
#pragma unroll
        for (int r = 0; r < S::kRows; r += 16) {
            Chunk<T> xv[S::kBlocksK];
#pragma unroll
            for (int j = 0; j < S::kBlocksK; ++j) xv[j] = operand<T, S::kPitchK>(from + kX, r, wave_k + j * 32, lane);
            // (of fp16 the second part is bf16: as fp16 it would be among the smallest numbers; x loses 2^-9 of 2^-12 in that product)
            constexpr bool kOther = std::is_same<T, _Float16>::value && PARTS == 2;
            Chunk<__bf16> xb[S::kBlocksK];
            if (kOther)
#pragma unroll
                for (int j = 0; j < S::kBlocksK; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) xb[j].v[e] = (__bf16)(float)xv[j].v[e];
            // the small parts first; three of them one after the other (their operands together would take too many registers)
            constexpr int kAtOnce = PARTS == 3 ? 1 : PARTS;
#pragma unroll
            for (int last = PARTS; last > 0; last -= kAtOnce) {
                Chunk<T> g[kAtOnce][S::kBlocksN];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
                    for (int i = 0; i < S::kBlocksN; ++i)
                        g[k][i] = operand<T, S::kPitchN>(from + (last - 1 - k) * S::kImageN, r, wave_n + i * 32, lane);
#pragma unroll
                for (int i = 0; i < S::kBlocksN; ++i)
#pragma unroll
                    for (int j = 0; j < S::kBlocksK; ++j)
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            if (kOther && k == 0) acc[i][j] = multiply(__builtin_bit_cast(Chunk<__bf16>, g[k][i]), xb[j], acc[i][j]);
                            else acc[i][j] = multiply(g[k][i], xv[j], acc[i][j]);
                        }
            }
        }
    };
    if (first < end) ask(first);
    if constexpr (S::kSkinny) {
        // W^T as operands: of channels k 32 .. block (k32, half a, n32) gives lane row r = lane mod 16 channel 8 (r / 4) + 4 a + r mod 4 and
        // 8 channels n, so that a lane's two results of four are eight neighbouring channels
        char* weights = lds + kStage;
        for (int f = wave; f < S::kBN * S::kBK / 512; f += 4) {
            const int n32 = f % (S::kBN / 32), a = f / (S::kBN / 32) & 1, k32 = f / (S::kBN / 32) >> 1, r = lane & 15;
            const int kk = k32 * 32 + 8 * (r >> 2) + 4 * a + (r & 3), nn = n32 * 32 + 8 * (lane >> 4);
            Chunk<T> v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v.v[j] = d.d_x && kk < d.K && nn + j < d.N ? ((const T*)d.w)[(long long)(nn + j) * d.K + kk] : (T)0.0f;
            *(Chunk<T>*)(weights + f * 1024 + lane * 16) = v;
        }
        constexpr int kGroups = S::kRows / 16, kPer = 4 / kGroups;   // groups of 16 positions; waves of a group
        const int r = wave % kGroups * 16 + (lane & 15);
        T* dx_at = (T*)d.d_x + (first + r) * d.xs + 8 * (lane >> 4);
        for (long long p0 = first; p0 < end; p0 += S::kRows) {
            put(lds, p0);
            __syncthreads();
            if (p0 + S::kRows < end) ask(p0 + S::kRows);
            if (multiplies) multiply_all(lds);
            if (d.d_x) {
                Chunk<T> g[S::kBN / 32];
#pragma unroll
                for (int i = 0; i < S::kBN / 32; ++i) g[i] = *(const Chunk<T>*)(lds + r * S::kPitchN + i * 64 + (lane >> 4) * 16);
#pragma unroll
                for (int kb = 0; kb < S::kBK / 32; kb += kPer) {
                    const int k32 = kb + wave / kGroups;
                    if (k32 * 32 >= S::kBK) continue;
                    f32x4 res[2] = {};
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int i = 0; i < S::kBN / 32; ++i)
                            res[a] = multiply16(*(const Chunk<T>*)(weights + ((k32 * 2 + a) * (S::kBN / 32) + i) * 1024 + lane * 16), g[i], res[a]);
                    Chunk<T> out;
#pragma unroll
                    for (int j = 0; j < 8; ++j) out.v[j] = (T)res[j >> 2][j & 3];
                    const int kk = k32 * 32 + 8 * (lane >> 4);
                    store_chunk<WHOLE>(dx_at + k32 * 32, p0 + r < end ? d.K - kk : 0, out);
                }
            }
            dx_at += S::kRows * d.xs;
            __syncthreads();
        }
    } else {
        if (first < end) {
            put(lds, first);
            if (first + S::kRows < end) ask(first + S::kRows);
        }
        __syncthreads();
        const bool early = wave < S::kWaves / 2;
        int buffer = 0;
        for (long long p0 = first; p0 < end; p0 += S::kRows) {
            char *from = lds + buffer * kStage, *to = lds + (buffer ^ 1) * kStage;
            const long long next = p0 + S::kRows;
            if (early && multiplies) multiply_all(from);
            if (next < end) {
                put(to, next);
                if (next + S::kRows < end) ask(next + S::kRows);
            }
            if (!early && multiplies) multiply_all(from);
            __syncthreads();
            buffer ^= 1;
        }
    }
    if (multiplies) {
        float* out = d.parts + (long long)split * d.N * d.K;
#pragma unroll
        for (int i = 0; i < S::kBlocksN; ++i)
#pragma unroll
            for (int j = 0; j < S::kBlocksK; ++j) {
                const int kk = k0 + wave_k + j * 32 + l32;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int nn = n0 + wave_n + i * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
                    if (kk < d.K && nn < d.N) out[(long long)nn * d.K + kk] = acc[i][j][e];
                }
            }
    }
    if (d.d_bias && k0 == 0) {
        float* sums = (float*)lds;   // [kDownN][BN]
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[rn * S::kBN + cn * 8 + j] = bias[j];
        __syncthreads();
        for (int c = threadIdx.x; c < S::kBN; c += S::kThreadsOf) {
            if (n0 + c >= d.N) continue;
            float sum = 0.0f;
            for (int r = 0; r < kDownN; ++r) sum += sums[r * S::kBN + c];
            d.bias_parts[(long long)split * d.N + n0 + c] = sum;
        }
    }
}

// Calls f with the shape of the gradients' kernel.
template <class F>
void with_back_shape(const Parts& p, bool skinny, F&& f)
{
    if (!skinny) {
        if (p.bk == 128) f(BackShape<128, 128, 2, 2, 32, false>());
        else if (p.bk == 256) f(BackShape<128, 256, 1, 4, 32, false>());
        else f(BackShape<128, 512, 1, 8, 32, false>());
    } else if (p.bn == 64) {
        if (p.bk == 32) f(BackShape<64, 32, 2, 1, 64, true>());
        else if (p.bk == 64) f(BackShape<64, 64, 2, 2, 64, true>());
        else f(BackShape<64, 128, 2, 2, 64, true>());
    } else {
        if (p.bk == 32) f(BackShape<128, 32, 4, 1, 64, true>());
        else if (p.bk == 64) f(BackShape<128, 64, 4, 1, 64, true>());
        else f(BackShape<128, 128, 2, 2, 32, true>());
    }
}

template <class T, bool WHOLE>
hipError_t launch_back(int act, const BackDev& d, const Parts& p, bool skinny, hipStream_t s)
{
    hipError_t e = hipSuccess;
    with_act_of(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        with_back_shape(p, skinny, [&](auto shape) {
            using S = decltype(shape);
            auto go = [&](auto kernel, int kLds) {
                if (kLds > 65536) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);   // (the same from every thread)
                if (e == hipSuccess)
                    hipLaunchKernelGGL(kernel, dim3((unsigned)(d.tiles_n * d.tiles_k * p.splits)), dim3(S::kThreadsOf), kLds, s, d);
            };
            auto with = [&](auto parts) {
                constexpr int N = decltype(parts)::value;
                go(linear_back_kernel<T, A, N, WHOLE, S>, S::lds(N));
            };
            if constexpr (A == LP_ACT_NONE || A == LP_ACT_RELU) {   // (d_z is d_y, or 0)
                with(std::integral_constant<int, 1>());
            } else if constexpr (std::is_same<T, __bf16>::value) {
                with(std::integral_constant<int, 3>());
            } else {
                with(std::integral_constant<int, 2>());
            }
        });
    });
    return e;
}

}  // namespace


}  // namespace linear
}  // namespace lp
