// Products of positions with a weight matrix in tiles, for all types and sizes, and d_x from d_y and what the forward kept.
#include "lp_linear.h"

namespace lp {
namespace linear {

namespace {

// ---- tiles -----------------------------------------------------------------------------------------------------
//
// A workgroup of four waves makes BP positions x BN channels.  A step is 128 bytes of channels of both operands, staged through
// registers into one of two LDS buffers while the other one is multiplied.  Latency bounds it where there are few tiles (a step of 16-bit types takes some
// 0.6 us then, of fp32 2), fp32 matrix instructions for large fp32 products (20000 x 1024 -> 1024 with GELU: 400 us, 0.1 PFLOP/s, 2.5 rounds of tiles).  Chunks lie in LDS as
// chunk_at says.
template <int BP, int BN>
struct TileShape {
    static constexpr int kWavesN = BN >= 128 ? 2 : 1, kWavesP = 4 / kWavesN;
    static constexpr int kP = BP / kWavesP, kN = BN / kWavesN;          // of a wave
    static constexpr int kBlocksP = kP / 32, kBlocksN = kN / 32;
    static constexpr int kPitch = kN + 4;                               // floats of a position's row while results are turned over
    static constexpr int kStage = (BP + BN) * 128;                      // bytes of a step
    static constexpr int kLds = 2 * kStage > 4 * 32 * kPitch * 4 ? 2 * kStage : 4 * 32 * kPitch * 4;
};

// Few tiles with long sums leave most of the chip idle and wait for the memory at every step: their steps are divided among workgroups (kPart), which
// leave their sums as the lanes hold them, and a second kernel (kJoin) adds these up and finishes them.
enum Mode { kWhole, kPart, kJoin };

template <class T, int ACT, bool BACK, bool WHOLE, int BP, int BN, Mode MODE>
__global__ __launch_bounds__(kThreads, 2) void linear_tile_kernel(LinearDev d)
{
    using S = TileShape<BP, BN>;
    constexpr int E = kChunk<T>;
    constexpr int kLoadsA = BP * 8 / kThreads, kLoadsW = BN * 8 / kThreads;
    __shared__ alignas(16) char lds[S::kLds];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
    const int wave_p = wave / S::kWavesN * S::kP, wave_n = wave % S::kWavesN * S::kN;
    const int c8 = threadIdx.x & 7, row = threadIdx.x >> 3;
    const long long tiles = d.tiles_p * d.tiles_n * (MODE == kPart ? d.splits : 1), rounds = (tiles + 7) / 8 * 8;
    for (long long b = blockIdx.x; b < rounds; b += gridDim.x) {
        const long long item = tile_of(b, tiles), tile = MODE == kPart ? item / d.splits : item;
        if (item >= tiles) continue;
        const long long p0 = tile / d.tiles_n * BP;
        const int n0 = (int)(tile % d.tiles_n) * BN;
        f32x16 acc[S::kBlocksN][S::kBlocksP] = {};
        // a part's sums: four of a lane's at a time, as the lanes hold them
        constexpr int kFours = S::kBlocksN * S::kBlocksP * 4;
        auto part = [&](long long k, int v) { return (f32x4*)d.parts + (k * kFours + v) * kThreads + threadIdx.x; };
        if constexpr (MODE == kJoin) {
            for (int k = 0; k < d.splits; ++k)
#pragma unroll
                for (int v = 0; v < kFours; ++v) {
                    const f32x4 sum = *part(tile * d.splits + k, v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[v / 4 / S::kBlocksP][v / 4 % S::kBlocksP][v % 4 * 4 + j] += sum[j];
                }
        } else {
            // (two steps are asked for ahead: where there are few tiles nothing else hides the memory's latency)
            struct Staged {
                Chunk<T> a[kLoadsA], pre[BACK && ACT != LP_ACT_NONE ? kLoadsA : 1], w[kLoadsW];
            } staged[2];
            // (only the last step can meet the end of a row: moving what is left of one waits for every piece)
            auto ask_as = [&](auto all, int step, Staged& to) {
                constexpr bool kAll = decltype(all)::value;
                const int k = step * (8 * E) + c8 * E;
#pragma unroll
                for (int u = 0; u < kLoadsA; ++u) {
                    const long long p = p0 + row + u * 32;
                    const int count = p < d.P ? d.K - k : 0;
                    to.a[u] = load_chunk<kAll>((const T*)d.a + p * d.as + k, count);
                    if (BACK && ACT != LP_ACT_NONE) to.pre[u] = load_chunk<kAll>((const T*)d.pre + p * d.K + k, count);
                }
#pragma unroll
                for (int u = 0; u < kLoadsW; ++u) {
                    const int n = n0 + row + u * 32;
                    to.w[u] = load_chunk<kAll>((const T*)d.w + n * d.ws + k, n < d.N ? d.K - k : 0);
                }
            };
            auto ask = [&](int step, Staged& to) {
                if (WHOLE || (step + 1) * (8 * E) <= d.K) ask_as(std::true_type(), step, to);
                else ask_as(std::false_type(), step, to);
            };
            auto put = [&](int buffer, const Staged& from) {
                char* to = lds + buffer * S::kStage;
#pragma unroll
                for (int u = 0; u < kLoadsA; ++u) {
                    Chunk<T> v = from.a[u];
                    if (BACK && ACT != LP_ACT_NONE) v = gradient<ACT>(from.a[u], from.pre[u]).part[0];
                    *(Chunk<T>*)(to + chunk_at(row + u * 32, c8)) = v;
                }
#pragma unroll
                for (int u = 0; u < kLoadsW; ++u) *(Chunk<T>*)(to + BP * 128 + chunk_at(row + u * 32, c8)) = from.w[u];
            };
            const int all_steps = (d.K + 8 * E - 1) / (8 * E), start = MODE == kPart ? (int)(item % d.splits) * d.split_steps : 0;
            const int steps = MODE == kPart ? min(d.split_steps, all_steps - start) : all_steps;
            auto multiply_all = [&](const char* from) {
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
            };
            ask(start, staged[0]);
            if (steps > 1) ask(start + 1, staged[1]);
            put(0, staged[0]);
            __syncthreads();
            for (int first = 0; first < steps; first += 2) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int s = first + u;
                    if (s >= steps) break;
                    if (s + 2 < steps) ask(start + s + 2, staged[u]);
                    multiply_all(lds + u * S::kStage);
                    if (s + 1 < steps) put(u ^ 1, staged[u ^ 1]);
                    __syncthreads();
                }
            }
        }
        if constexpr (MODE == kPart) {
#pragma unroll
            for (int v = 0; v < kFours; ++v) {
                const f32x16& from = acc[v / 4 / S::kBlocksP][v / 4 % S::kBlocksP];
                *part(item, v) = f32x4{from[v % 4 * 4], from[v % 4 * 4 + 1], from[v % 4 * 4 + 2], from[v % 4 * 4 + 3]};
            }
            continue;
        }
        float* turn = (float*)lds + wave * 32 * S::kPitch;
        if (WHOLE || n0 + wave_n + S::kN <= d.N) finish<T, ACT, BACK, true, S::kBlocksP, S::kBlocksN>(d, acc, turn, p0 + wave_p, n0 + wave_n, lane);
        else finish<T, ACT, BACK, false, S::kBlocksP, S::kBlocksN>(d, acc, turn, p0 + wave_p, n0 + wave_n, lane);
        __syncthreads();   // (the next tile's first step lies where results were)
    }
}

template <class T, int ACT, bool BACK>
void tiles(LinearDev d, bool whole, hipStream_t s)
{
    auto launch = [&](auto bn, auto mode, auto all) {
        constexpr int BN = decltype(bn)::value;
        constexpr Mode M = decltype(mode)::value;
        d.tiles_p = (d.P + kTileP - 1) / kTileP;
        d.tiles_n = (d.N + BN - 1) / BN;
        const long long items = d.tiles_p * d.tiles_n * (M == kPart ? d.splits : 1);
        hipLaunchKernelGGL((linear_tile_kernel<T, ACT, BACK, decltype(all)::value, kTileP, BN, M>), dim3(grid_of((items + 7) / 8 * 8)), dim3(kThreads), 0, s, d);
    };
    auto go = [&](auto bn) {
        auto with = [&](auto mode) { whole ? launch(bn, mode, std::true_type()) : launch(bn, mode, std::false_type()); };
        if (d.splits > 1) {
            with(std::integral_constant<Mode, kPart>());
            with(std::integral_constant<Mode, kJoin>());
        } else {
            with(std::integral_constant<Mode, kWhole>());
        }
    };
    const int bn = tile_channels(d.N);
    if (bn == 32) go(std::integral_constant<int, 32>());
    else if (bn == 64) go(std::integral_constant<int, 64>());
    else go(std::integral_constant<int, 128>());
}

}  // namespace

// Tiles of 128 x 128 results, narrower ones where there are few channels.
void launch_tiles(int dtype, int act, bool back, LinearDev d, hipStream_t s)
{
    const bool w = whole(d, dtype);
    with_act_of(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        if (dtype == LP_BF16) back ? tiles<__bf16, A, true>(d, w, s) : tiles<__bf16, A, false>(d, w, s);
        else if (dtype == LP_F16) back ? tiles<_Float16, A, true>(d, w, s) : tiles<_Float16, A, false>(d, w, s);
        else back ? tiles<float, A, true>(d, w, s) : tiles<float, A, false>(d, w, s);
    });
}

}  // namespace linear
}  // namespace lp
