// Products of positions with a weight matrix in 16-bit types that make more than 128 channels.
#include "lp_linear.h"

namespace lp {
namespace linear {

namespace {

constexpr int kWideP = 128, kWideN = 256;
// ---- wide tiles (16-bit types) ---------------------------------------------------------------------------------
//
// Four waves make 128 positions x 256 channels, each of them all positions and 64 channels.  The positions go through LDS (two buffers), the
// weights, of which no two waves need the same, straight to registers, from a copy in the order of the matrix instructions' operands
// (blocks of 32 channels x 16 summed ones, 16 bytes a lane): for a step of 64 summed channels the matrix cores take 1024 cycles, LDS (128 bytes a
// cycle) 640, the cache (64 bytes a cycle) 512.  Two workgroups share a compute unit, so that one's products can run under the other's epilogue.
// Measured: 65536 x 2048 -> 512 in bf16 148 us (0.93 PFLOP/s; matrix cores busy 53 % of the time, waits for barriers and memory 30 %), 65536 x 512 -> 2048
// 206 us bare, 225 with GELU, 238 with z kept too (0.6 GB; a copy's rate would be 122).
struct WideShape {
    static constexpr int kBuffer = kWideP * 128, kTurn = 4 * 32 * 68 * 4;
    static constexpr int kLds = 2 * kBuffer > kTurn ? 2 * kBuffer : kTurn;
};

// The weights as operands: block (i, j) holds rows 32 i .. and columns 16 j .., zeros behind the last ones.  TURNED: rows are W's columns.
template <class T, bool TURNED>
__global__ __launch_bounds__(kThreads) void linear_pack_kernel(const T* w, int rows, int cols, int pitch, Chunk<T>* out)
{
    const int lane = threadIdx.x & 63, across = wide_blocks(cols);
    const long long blocks = (long long)((rows + 31) / 32) * across;
    for (long long b = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); b < blocks; b += (long long)gridDim.x * (kThreads / 64)) {
        const int r = (int)(b / across) * 32 + (lane & 31), c = (int)(b % across) * 16 + (lane >> 5) * 8;
        Chunk<T> v;
        if (TURNED) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v.v[j] = r < rows && c + j < cols ? w[(long long)(c + j) * pitch + r] : (T)0.0f;
        } else {
            v = load_chunk<false>(w + (long long)r * pitch + c, r < rows ? cols - c : 0);
        }
        out[b * 64 + lane] = v;
    }
}

template <class T, int ACT, bool BACK, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void linear_wide_kernel(LinearDev d)
{
    __shared__ alignas(16) char lds[WideShape::kLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
    const int c8 = threadIdx.x & 7, row = threadIdx.x >> 3;
    const long long tiles = d.tiles_p * d.tiles_n, rounds = (tiles + 7) / 8 * 8;
    const int across = wide_blocks(d.K), steps = across / 4, last_block = (d.N + 31) / 32 - 1;
    for (long long b = blockIdx.x; b < rounds; b += gridDim.x) {
        const long long tile = tile_of(b, tiles);
        if (tile >= tiles) continue;
        const long long p0 = tile / d.tiles_n * kWideP;
        const int n0 = (int)(tile % d.tiles_n) * kWideN + wave * 64;
        const T* at[4];
        int rows_in = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long p = p0 + row + u * 32;
            at[u] = (const T*)d.a + p * d.as + c8 * 8;
            rows_in |= (p < d.P) << u;
        }
        Chunk<T> staged[4];
        auto ask = [&](int step) {
            const int k = step * 64;
            const int count = d.K - k - c8 * 8;
            if (WHOLE || k + 64 <= d.K) {   // (only the last step can meet the end of a row)
#pragma unroll
                for (int u = 0; u < 4; ++u) staged[u] = load_chunk<true>(at[u] + k, rows_in >> u & 1 ? count : 0);
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u) staged[u] = load_chunk<false>(at[u] + k, rows_in >> u & 1 ? count : 0);
            }
        };
        auto put = [&](int buffer) {
#pragma unroll
            for (int u = 0; u < 4; ++u) *(Chunk<T>*)(lds + buffer * WideShape::kBuffer + chunk_at(row + u * 32, c8)) = staged[u];
        };
        const Chunk<T>* w_at[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w_at[i] = (const Chunk<T>*)d.w + (long long)min((n0 >> 5) + i, last_block) * across * 64 + lane;
        Chunk<T> w[4][2], a[2][4];
        auto ask_w = [&](int k16, Chunk<T> (&to)[2]) {
            k16 = min(k16, across - 1);   // (behind the last step: not used)
#pragma unroll
            for (int i = 0; i < 2; ++i) to[i] = w_at[i][k16 * 64];
        };
        auto get = [&](int buffer, int q, Chunk<T> (&to)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = *(const Chunk<T>*)(lds + buffer * WideShape::kBuffer + chunk_at(i * 32 + l32, 2 * q + h));
        };
        f32x16 acc[2][4] = {};
        ask(0);
#pragma unroll
        for (int q = 0; q < 4; ++q) ask_w(q, w[q]);
        put(0);
        if (steps > 1) ask(1);
        __syncthreads();
        for (int s = 0; s < steps; ++s) {
            const int buffer = s & 1;
            get(buffer, 0, a[0]);
            if (s + 1 < steps) put(buffer ^ 1);
            if (s + 2 < steps) ask(s + 2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q < 3) get(buffer, q + 1, a[(q + 1) & 1]);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = multiply(w[q][i], a[q & 1][j], acc[i][j]);
                ask_w((s + 1) * 4 + q, w[q]);
                __builtin_amdgcn_sched_barrier(0);
            }
            __syncthreads();
        }
        if (WHOLE || n0 + 64 <= d.N) finish<T, ACT, BACK, true, 4, 2>(d, acc, (float*)lds + wave * 32 * 68, p0, n0, lane);
        else finish<T, ACT, BACK, false, 4, 2>(d, acc, (float*)lds + wave * 32 * 68, p0, n0, lane);
        __syncthreads();   // (the next tile's first step lies where results were)
    }
}

template <class T, int ACT, bool BACK>
void wide_tiles(const LinearDev& d, bool whole, hipStream_t s)
{
    const dim3 grid(grid_of((d.tiles_p * d.tiles_n + 7) / 8 * 8));
    if (whole) hipLaunchKernelGGL((linear_wide_kernel<T, ACT, BACK, true>), grid, dim3(kThreads), 0, s, d);
    else hipLaunchKernelGGL((linear_wide_kernel<T, ACT, BACK, false>), grid, dim3(kThreads), 0, s, d);
}

}  // namespace

void launch_pack(int dtype, bool turned, const void* w, int rows, int cols, int pitch, void* out, hipStream_t s)
{
    const dim3 grid(grid_of(((long long)(rows + 31) / 32 * wide_blocks(cols) + 3) / 4));
    auto go = [&](auto kernel, auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, (const T*)w, rows, cols, pitch, (Chunk<T>*)out);
    };
    if (dtype == LP_BF16) turned ? go(linear_pack_kernel<__bf16, true>, __bf16()) : go(linear_pack_kernel<__bf16, false>, __bf16());
    else turned ? go(linear_pack_kernel<_Float16, true>, _Float16()) : go(linear_pack_kernel<_Float16, false>, _Float16());
}

void launch_wide(int dtype, int act, bool back, LinearDev d, hipStream_t s)
{
    d.tiles_p = (d.P + kWideP - 1) / kWideP;
    d.tiles_n = (d.N + kWideN - 1) / kWideN;
    const bool w = whole(d, dtype);
    if (back) {
        if (dtype == LP_BF16) wide_tiles<__bf16, LP_ACT_NONE, true>(d, w, s);
        else wide_tiles<_Float16, LP_ACT_NONE, true>(d, w, s);
        return;
    }
    with_act_of(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        if (dtype == LP_BF16) wide_tiles<__bf16, A, false>(d, w, s);
        else wide_tiles<_Float16, A, false>(d, w, s);
    });
}

}  // namespace linear
}  // namespace lp
