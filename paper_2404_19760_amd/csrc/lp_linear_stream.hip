// Products of positions of few channels with a weight matrix: up to 256 bytes of summed channels, up to 128 channels made.
//
// Memory bounds them (32 -> 64 channels in fp32: 384 bytes and 4096 operations a position), so nothing is shared between waves but the
// weights, which lie in LDS as the matrix instructions' operands for as long as the workgroup lives: a wave takes 32 positions at a time,
// asks for the next 32 before it multiplies, and never waits for another wave.  The positions' channels go straight to registers: of a row's
// 16-byte chunks lanes 0 .. 31 ask for the even ones, lanes 32 .. 63 for the odd ones.
//
// Rows are taken in steps of 64 bytes, two pairs of chunks (each step is a kernel of its own; what a row leaves of its last one is multiplied as zeros):
// 131979 x 48 -> 128 in fp32 takes 39 us with six pairs and 46 with eight, x 36 36 and, with the five pairs that would do, 31; x 72 -> 128 in
// fp16 18.4 and 18.1.
// Measured: 160^3 x 32 -> 64 in fp32 302 us for 1.57 GB (5.2 TB/s; through LDS with a barrier a step 373), 131979 x 72 -> 96 in fp16 with residual
// 20 us for 70 MB, -> 97 30 us: rows of 194 bytes share the 64-byte lines that they are stored to.
#include "lp_linear.h"

namespace lp {
namespace linear {

namespace {

constexpr int kTurn = 32 * 36 * 4;   // bytes in which a wave turns over 32 x 32 results

// PAIRS: pairs of chunks of a row; BLOCKS: of 32 channels.  BACK: d_x from d_y and pre, the weights are W's columns.
template <class T, int ACT, bool BACK, bool WHOLE, int PAIRS, int BLOCKS>
__global__ __launch_bounds__(kThreads, PAIRS * BLOCKS > 16 ? 2 : 3) void linear_stream_kernel(LinearDev d)
{
    constexpr int E = kChunk<T>;
    constexpr bool kSlope = BACK && ACT != LP_ACT_NONE;
    __shared__ alignas(16) char lds[PAIRS * BLOCKS * 1024 + 4 * kTurn];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
    const long long step = (long long)gridDim.x * 128;
    const int n0 = blockIdx.y * (BLOCKS * 32);   // the first of its channels
    long long p0 = (long long)blockIdx.x * 128 + wave * 32;
    const T *a_at = (const T*)d.a + (p0 + l32) * d.as + h * E, *pre_at = (const T*)d.pre + (p0 + l32) * d.K + h * E;
    Chunk<T> a[PAIRS], pre[kSlope ? PAIRS : 1];
    auto ask = [&](long long p) {
#pragma unroll
        for (int f = 0; f < PAIRS; ++f) {
            const int count = p + l32 < d.P ? d.K - (2 * f + h) * E : 0;
            if (WHOLE || (2 * f + 2) * E <= d.K) {   // (the same for all lanes)
                a[f] = load_chunk<true>(a_at + 2 * f * E, count);
                if (kSlope) pre[f] = load_chunk<true>(pre_at + 2 * f * E, count);
            } else {
                a[f] = load_chunk<false>(a_at + 2 * f * E, count);
                if (kSlope) pre[f] = load_chunk<false>(pre_at + 2 * f * E, count);
            }
        }
        a_at += step * d.as;
        pre_at += step * d.K;
    };
    if (p0 < d.P) ask(p0);
    for (int b = wave; b < PAIRS * BLOCKS; b += 4) {
        const int n = n0 + b / PAIRS * 32 + l32, k = (2 * (b % PAIRS) + h) * E;
        Chunk<T> w;
        if (BACK) {
#pragma unroll
            for (int j = 0; j < E; ++j) w.v[j] = n < d.N && k + j < d.K ? ((const T*)d.w)[(k + j) * d.ws + n] : (T)0.0f;
        } else {
            w = load_chunk<false>((const T*)d.w + n * d.ws + k, n < d.N ? d.K - k : 0);
        }
        *(Chunk<T>*)(lds + b * 1024 + lane * 16) = w;
    }
    __syncthreads();
    float* turn = (float*)(lds + PAIRS * BLOCKS * 1024 + wave * kTurn);
    for (; p0 < d.P; p0 += step) {
        Chunk<T> av[PAIRS];
#pragma unroll
        for (int f = 0; f < PAIRS; ++f) av[f] = kSlope ? gradient<ACT>(a[f], pre[f]).part[0] : a[f];
        // (the residual of two blocks of channels is on its way while others are finished)
        Chunk<T> added[2][kFinishTimes<T, 1>];
        auto residual = [&](int n, Chunk<T> (&to)[kFinishTimes<T, 1>]) {
            if (WHOLE || n + 32 <= d.N) ask_residual<T, true, 1>(d, p0, n, lane, to);
            else ask_residual<T, false, 1>(d, p0, n, lane, to);
        };
        if (!BACK && d.res) {
            residual(n0, added[0]);
            if (BLOCKS > 1) residual(n0 + 32, added[1]);
        }
        if (p0 + step < d.P) ask(p0 + step);
        f32x16 acc[BLOCKS] = {};
#pragma unroll
        for (int f = 0; f < PAIRS; ++f)
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) acc[i] = multiply(*(const Chunk<T>*)(lds + (i * PAIRS + f) * 1024 + lane * 16), av[f], acc[i]);
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            if (n0 + i * 32 >= d.N) break;
            const f32x16 one[1][1] = {{acc[i]}};
            if (WHOLE || n0 + i * 32 + 32 <= d.N) finish<T, ACT, BACK, true, 1, 1>(d, one, turn, p0, n0 + i * 32, lane, &added[i & 1]);
            else finish<T, ACT, BACK, false, 1, 1>(d, one, turn, p0, n0 + i * 32, lane, &added[i & 1]);
            if (!BACK && d.res && i + 2 < BLOCKS) residual(n0 + (i + 2) * 32, added[i & 1]);
        }
    }
}

template <class T, int ACT, bool BACK, int PAIRS, int BLOCKS>
void go(const LinearDev& d, bool whole, int n_cu, hipStream_t s)
{
    const long long groups = (d.P + 127) / 128, most = (PAIRS * BLOCKS > 16 ? 2ll : 3ll) * n_cu;
    const dim3 grid((unsigned)(groups < most ? groups : most), (d.N + BLOCKS * 32 - 1) / (BLOCKS * 32));
    if (whole) hipLaunchKernelGGL((linear_stream_kernel<T, ACT, BACK, true, PAIRS, BLOCKS>), grid, dim3(kThreads), 0, s, d);
    else hipLaunchKernelGGL((linear_stream_kernel<T, ACT, BACK, false, PAIRS, BLOCKS>), grid, dim3(kThreads), 0, s, d);
}

template <class T, int ACT, bool BACK>
void stream(const LinearDev& d, bool whole, int n_cu, hipStream_t s)
{
    auto blocks = [&](auto pairs) {
        constexpr int P = decltype(pairs)::value;
        if (d.N <= 32) go<T, ACT, BACK, P, 1>(d, whole, n_cu, s);
        else if (d.N <= 64) go<T, ACT, BACK, P, 2>(d, whole, n_cu, s);
        // Up to 128 channels, few positions (below eight groups of 128 for each compute unit): two workgroups share the channels and both read the
        // positions.  Twice as many workgroups, with half the products and results of a group each, fill the chip better: x 72 -> 128 in fp16, 20000
        // positions 6.1 us instead of 8.1, 131979 18.4 instead of 20.7 (with residual 24 and 32).  With more of them reading once is faster:
        // 400000 positions 39 us instead of 41, x 128 50 instead of 57, 1 million 109 instead of 125 (not with a residual: 67 instead of 52).
        else if ((d.P + 127) / 128 < 8 * n_cu) go<T, ACT, BACK, P, 2>(d, whole, n_cu, s);
        else go<T, ACT, BACK, P, 4>(d, whole, n_cu, s);
    };
    const int bytes = d.K * (int)sizeof(T);
    if (bytes <= 64) blocks(std::integral_constant<int, 2>());
    else if (bytes <= 128) blocks(std::integral_constant<int, 4>());
    else if (bytes <= 192) blocks(std::integral_constant<int, 6>());
    else blocks(std::integral_constant<int, 8>());
}

}  // namespace

void launch_stream(int dtype, int act, bool back, const LinearDev& d, int n_cu, hipStream_t s)
{
    const bool w = whole(d, dtype);
    with_act_of(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        if (dtype == LP_BF16) stream<__bf16, A, false>(d, w, n_cu, s);
        else if (dtype == LP_F16) stream<_Float16, A, false>(d, w, n_cu, s);
        else back ? stream<float, A, true>(d, w, n_cu, s) : stream<float, A, false>(d, w, n_cu, s);
    });
}

}  // namespace linear
}  // namespace lp
