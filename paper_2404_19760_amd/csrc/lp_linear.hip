// Products of positions' channels with a weight matrix, with bias, activation and residual in the epilogue, and their gradients.
//
//     z = x W^T + b,   y = act(z) + r;   d_z = d_y act'(z),   d_x = d_z W,   d_W += d_z^T x,   d_b += sum d_z
//
// What bounds it: memory where a grid's positions have few channels (32 -> 64 channels in fp32: 384 bytes for 4096 operations a position), the
// matrix cores for blocks of some hundred channels, latency for single tokens.
//
// Everything moves in chunks of 16 bytes along the channels.  A 32 x 32 block of results is made from chunks the same way in all types: of two
// neighbouring chunks of a row lanes 0 .. 31 hold the first, lanes 32 .. 63 the second, and that is one 32x32x16 product in 16 bits and
// four 32x32x2 products in fp32 (the order of the channels in a sum does not matter as long as both operands have the same).
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "lp_lanes.h"
#include "lp_linear.h"

namespace lp {

using namespace linear;

namespace {

constexpr int kFewRows = 8;   // positions that a wave of the kernel without matrix cores makes, at most

// ---- few positions ---------------------------------------------------------------------------------------------
//
// A wave makes kOutputs channels of up to ROWS positions: lanes share the sum, 16 bytes of a weight's row each.  One position, 512 -> 2048 in bf16: 3.8 us,
// most of it a launch's.
constexpr int kOutputs = 2;
template <class T, int ACT, int ROWS>
__global__ __launch_bounds__(kThreads) void linear_rows_kernel(LinearDev d)
{
    constexpr int E = kChunk<T>;
    const int lane = threadIdx.x & 63, n0 = (blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * kOutputs, r0 = blockIdx.y * ROWS;
    if (n0 >= d.N) return;
    float sum[kOutputs][ROWS] = {};
    for (int k = lane * E; k < d.K; k += 64 * E) {
        Chunk<T> w[kOutputs], x[ROWS];
#pragma unroll
        for (int i = 0; i < kOutputs; ++i) w[i] = load_chunk<false>((const T*)d.w + (n0 + i) * d.ws + k, n0 + i < d.N ? d.K - k : 0);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) x[r] = load_chunk<false>((const T*)d.a + (r0 + r) * d.as + k, r0 + r < d.P ? d.K - k : 0);
#pragma unroll
        for (int i = 0; i < kOutputs; ++i)
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int j = 0; j < E; ++j) sum[i][r] = fmaf((float)w[i].v[j], (float)x[r].v[j], sum[i][r]);
    }
#pragma unroll
    for (int i = 0; i < kOutputs; ++i) lane_sums(sum[i], 64);
#pragma unroll
    for (int i = 0; i < kOutputs; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int n = n0 + i;
            if (lane != i * ROWS + r || n >= d.N || r0 + r >= d.P) continue;
            const float z = sum[i][r] + (d.bias ? d.bias[n] : 0.0f);
            if (d.keep) ((T*)d.keep)[(long long)(r0 + r) * d.N + n] = (T)z;
            float y = activate_as<ACT, T>(z);
            if (d.res) y += (float)((const T*)d.res)[(r0 + r) * d.rs + n];
            ((T*)d.out)[(r0 + r) * d.ys + n] = (T)y;
        }
}

// ---- gradients of the parameters in fp32 -----------------------------------------------------------------------
//
// A workgroup sums a part of the positions into 128 or 64 channels of d_z x 128 channels of x, with fp32 matrix instructions; both operands lie in LDS as
// they lie in memory, row by row, 32 positions in one of two buffers while the other one is multiplied and 64 more are on their way.
struct WeightDev {
    long long P;
    int K, N;
    long long xs, ys;
    const float *x, *dy, *pre;
    float *d_weight, *d_bias;
    float *parts, *bias_parts;   // [splits][N][K], [splits][N]; NULL: one split, into d_weight and d_bias
    long long chunk;             // positions of a part
    int tiles_n, tiles_k, splits;
};
constexpr int kWeightTile = 128, kWeightRows = 32;

// BN: channels of d_z (the four waves make 64 x 64 or 32 x 64 of the sums each)
template <int ACT, int BN>
__global__ __launch_bounds__(kThreads, 2) void linear_weight_kernel(WeightDev d)
{
    constexpr int E = 4, kRows = kWeightRows, kPitchN = BN * 4 + 64, kPitchK = kWeightTile * 4 + 64, kBlocks = BN / 64;
    constexpr int kAcrossN = BN / E, kDownN = kThreads / kAcrossN, kLoadsN = kRows / kDownN;
    constexpr int kAcrossK = kWeightTile / E, kDownK = kThreads / kAcrossK, kLoadsK = kRows / kDownK;
    constexpr int kImage = kRows * kPitchN, kStage = kImage + kRows * kPitchK;
    __shared__ alignas(16) char lds[2 * kStage];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
    const int cn = threadIdx.x % kAcrossN, rn = threadIdx.x / kAcrossN, ck = threadIdx.x % kAcrossK, rk = threadIdx.x / kAcrossK;
    const int wave_n = (wave >> 1) * (BN / 2), wave_k = (wave & 1) * 64;
    const int tiles = d.tiles_n * d.tiles_k, split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int n0 = tile / d.tiles_k * BN, k0 = tile % d.tiles_k * kWeightTile;
    const long long first = split * d.chunk, end = min(d.P, first + d.chunk);
    struct Staged {
        Chunk<float> dy[kLoadsN], pre[kLoadsN], x[kLoadsK];
    } staged[2];
    float bias[E] = {};
    const int n = n0 + cn * E, k = k0 + ck * E;
    const bool sum_bias = d.d_bias && k0 == 0;
    auto ask = [&](long long p0, Staged& to) {   // (behind the last position: zeros)
#pragma unroll
        for (int u = 0; u < kLoadsN; ++u) {
            const long long p = p0 + rn + u * kDownN;
            const int count = p < end ? d.N - n : 0;
            to.dy[u] = load_chunk<false>(d.dy + p * d.ys + n, count);
            if (ACT != LP_ACT_NONE) to.pre[u] = load_chunk<false>(d.pre + p * d.N + n, count);
        }
#pragma unroll
        for (int u = 0; u < kLoadsK; ++u) {
            const long long p = p0 + rk + u * kDownK;
            to.x[u] = load_chunk<false>(d.x + p * d.xs + k, p < end ? d.K - k : 0);
        }
    };
    auto put = [&](int buffer, const Staged& from) {
        char* to = lds + buffer * kStage;
#pragma unroll
        for (int u = 0; u < kLoadsN; ++u) {
            const Gradient<float> g = gradient<ACT>(from.dy[u], from.pre[u]);
            *(Chunk<float>*)(to + (rn + u * kDownN) * kPitchN + cn * 16) = g.part[0];
#pragma unroll
            for (int j = 0; j < E; ++j) bias[j] += g.v[j];
        }
#pragma unroll
        for (int u = 0; u < kLoadsK; ++u) *(Chunk<float>*)(to + kImage + (rk + u * kDownK) * kPitchK + ck * 16) = from.x[u];
    };
    f32x16 acc[kBlocks][2] = {};
    auto multiply_all = [&](const char* from) {
#pragma unroll
        for (int r = 0; r < kRows; r += 2) {
            float xv[2], g[kBlocks];
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) g[i] = *(const float*)(from + (r + h) * kPitchN + (wave_n + i * 32 + l32) * 4);
#pragma unroll
            for (int j = 0; j < 2; ++j) xv[j] = *(const float*)(from + kImage + (r + h) * kPitchK + (wave_k + j * 32 + l32) * 4);
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(g[i], xv[j], acc[i][j], 0, 0, 0);
        }
    };
    ask(first, staged[0]);
    ask(first + kRows, staged[1]);
    put(0, staged[0]);
    __syncthreads();
    for (long long p = first; p < end; p += 2 * kRows) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const long long at = p + u * kRows;
            if (at >= end) break;
            if (at + 2 * kRows < end) ask(at + 2 * kRows, staged[u]);
            multiply_all(lds + u * kStage);
            if (at + kRows < end) put(u ^ 1, staged[u ^ 1]);
            __syncthreads();
        }
    }
    if (d.d_weight) {
        float* out = d.parts ? d.parts + (long long)split * d.N * d.K : d.d_weight;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
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
        float* sums = (float*)lds;   // [kDownN][BN]
#pragma unroll
        for (int j = 0; j < E; ++j) sums[rn * BN + cn * E + j] = bias[j];
        __syncthreads();
        if (threadIdx.x < BN && n0 + (int)threadIdx.x < d.N) {
            float sum = 0.0f;
            for (int r = 0; r < kDownN; ++r) sum += sums[r * BN + threadIdx.x];
            const int nn = n0 + threadIdx.x;
            if (d.parts) d.bias_parts[(long long)split * d.N + nn] = sum;
            else d.d_bias[nn] += sum;
        }
    }
}

// out += the sum of its parts, in an order that depends on the sizes alone: a lane four values, `lanes` (a power of two) share the parts.
struct JoinDev {
    const float *parts, *bias_parts;
    float *out, *d_bias;
    long long count;
    int N, splits, lanes, bias_lanes;
};
__global__ __launch_bounds__(kThreads) void linear_join_kernel(JoinDev d)
{
    __shared__ f32x4 lds[kThreads];
    const int each = kThreads / d.lanes * 4, bias_each = kThreads / d.bias_lanes * 4;   // values of a workgroup
    const long long blocks = d.out ? (d.count + each - 1) / each : 0, all = blocks + (d.d_bias ? (d.N + bias_each - 1) / bias_each : 0);
    for (long long b = blockIdx.x; b < all; b += gridDim.x) {
        const bool weight = b < blocks;
        const int lanes = weight ? d.lanes : d.bias_lanes, across = kThreads / lanes, c = threadIdx.x % across, lane = threadIdx.x / across;
        const long long size = weight ? d.count : d.N, i = (weight ? b : b - blocks) * (across * 4) + c * 4;
        const float* from = (weight ? d.parts : d.bias_parts) + i;
        float* to = (weight ? d.out : d.d_bias) + i;
        const int in = (int)max(0ll, min(4ll, size - i));
        f32x4 sum = {};
        if (in == 4) {
#pragma unroll 4
            for (int s = lane; s < d.splits; s += lanes) {
                f32x4 v;
                __builtin_memcpy(&v, from + s * size, 16);
                sum += v;
            }
        } else {
            for (int s = lane; s < d.splits; s += lanes)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < in) sum[j] += from[s * size + j];
        }
        __syncthreads();   // (the sums before have been read)
        lds[threadIdx.x] = sum;
        __syncthreads();
        if (lane) continue;
        for (int s = 1; s < lanes; ++s) sum += lds[s * across + c];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < in) to[j] += sum[j];
    }
}
// Lanes that share the parts: as many as it takes to give every compute unit work.
int join_lanes(long long count, int splits)
{
    int lanes = 1;
    while (lanes < 64 && lanes * 2 <= splits && count * lanes < 512ll * kThreads * 4) lanes *= 2;
    return lanes;
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

// Parts: workgroups for all compute units, at least some steps each.
Parts parts_of(const Call& c, int n_cu)
{
    Parts p;
    p.bn = p.bk = kWeightTile;
    long long per_cu = 2, step = 32, least = 256;
    if (c.dtype == LP_F32) {
        if (c.N <= 64) p.bn = 64;
        least = 128;
    } else {
        if (c.K <= 128 && c.N <= 128) {
            p.bn = c.N <= 64 ? 64 : 128;
            p.bk = c.K <= 32 ? 32 : c.K <= 64 ? 64 : 128;
            per_cu = 3;
            step = 64;
            least = 64;
        } else {
            p.bk = c.K <= 128 ? 128 : c.K <= 256 ? 256 : 512;
            per_cu = p.bk == 512 ? 1 : 2;
        }
    }
    p.tiles_n = (c.N + p.bn - 1) / p.bn;
    p.tiles_k = (c.K + p.bk - 1) / p.bk;
    const long long tiles = (long long)p.tiles_n * p.tiles_k, target = (per_cu * n_cu + tiles - 1) / tiles;
    // (nor more sums of parts than twice what the positions hold: they are written and read again)
    const long long most = (c.P + least - 1) / least;
    const double light = 2.0 * c.P * (c.K + 2.0 * c.N) * dtype_bytes(c.dtype) / (4.0 * c.N * c.K);
    long long splits = target < most ? target : most;
    if ((double)splits > light) splits = (long long)light;
    if (splits < 1) splits = 1;
    p.chunk = ((c.P + splits - 1) / splits + step - 1) / step * step;
    if (p.chunk < step) p.chunk = step;
    p.splits = (int)((c.P + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    return p;
}

// The kernels of 16-bit types for products that make more than 128 channels, where there are tiles for some of the compute units.
bool is_wide(const Call& c, int channels) { return c.dtype != LP_F32 && channels > 128 && c.P >= 512; }
size_t packed_bytes(int rows, int cols) { return align256((size_t)((rows + 31) / 32) * wide_blocks(cols) * 1024); }
bool is_skinny(const Call& c) { return c.dtype != LP_F32 && c.K <= 128 && c.N <= 128; }

// How the general kernel divides long sums of few tiles: at least four steps (of 128 bytes) a part, some parts at most, for up to one workgroup and a
// half a compute unit.
struct Split {
    int splits, steps;
    size_t bytes;
};
Split split_of(const Call& c, int summed, int made, int n_cu)
{
    const int steps = (int)(((long long)summed * dtype_bytes(c.dtype) + 127) / 128), bn = tile_channels(made);
    const long long tiles = ((c.P + kTileP - 1) / kTileP) * ((made + bn - 1) / bn), room = 3ll * n_cu / 2 / (tiles > 0 ? tiles : 1);
    long long splits = steps / 4 < room ? steps / 4 : room;
    const int most = c.dtype == LP_F32 ? 8 : 4;   // (a step of fp32 takes 2 us, of 16 bits a third; adding up a part 1 to 2)
    if (splits > most) splits = most;
    Split s = {1, steps, 0};
    if (splits < 2) return s;
    s.steps = (int)((steps + splits - 1) / splits);
    s.splits = (steps + s.steps - 1) / s.steps;
    s.bytes = align256((size_t)tiles * s.splits * kTileP * bn * sizeof(float));
    return s;
}

struct Sizes {
    size_t weight, parts, bias_parts, dz, split;
    size_t all() const { return weight + parts + bias_parts + dz + split; }
};
Sizes sizes(const Call& c, int n_cu)
{
    const Parts p = parts_of(c, n_cu);
    const size_t E = 16 / dtype_bytes(c.dtype);
    const bool halves = c.dtype != LP_F32;
    Sizes s;
    s.weight = is_skinny(c) ? 0 : is_wide(c, c.K) ? packed_bytes(c.K, c.N) : align256((size_t)c.K * ((c.N + E - 1) / E * E) * dtype_bytes(c.dtype));
    s.parts = halves || p.splits > 1 ? align256((size_t)p.splits * c.N * c.K * sizeof(float)) : 0;
    s.bias_parts = halves || p.splits > 1 ? align256((size_t)p.splits * c.N * sizeof(float)) : 0;
    s.split = split_of(c, c.N, c.K, n_cu).bytes;
    s.dz = halves && !is_skinny(c) && c.act != LP_ACT_NONE ? align256((size_t)c.P * c.N * 2) : 0;
    return s;
}

lp_status launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LP_OK : fail(LP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// Bytes that a call moves of `channels` channels a position.
double bytes_of(const Call& c, double channels) { return (double)c.P * channels * dtype_bytes(c.dtype); }

lp_status aligned(int dtype, std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if ((uintptr_t)p % dtype_bytes(dtype)) return fail(LP_ERR_INVALID_ARG, "tensors must be aligned to their elements");
    return LP_OK;
}

template <class T>
void few_rows(const LinearDev& d, int act, hipStream_t s)
{
    dim3 grid((d.N + kThreads / 64 * kOutputs - 1) / (kThreads / 64 * kOutputs));
    if (d.P > kFewRows) grid.y = (unsigned)((d.P + kFewRows - 1) / kFewRows);
    with_act_of(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        if (d.P == 1) hipLaunchKernelGGL((linear_rows_kernel<T, A, 1>), grid, dim3(kThreads), 0, s, d);
        else if (d.P <= 4) hipLaunchKernelGGL((linear_rows_kernel<T, A, 4>), grid, dim3(kThreads), 0, s, d);
        else hipLaunchKernelGGL((linear_rows_kernel<T, A, kFewRows>), grid, dim3(kThreads), 0, s, d);
    });
}

// Which kernel makes a forward.
enum Way { kRowsWay, kStreamWay, kWideWay, kTileWay };
// Up to eight positions go to the kernel without matrix cores.  Some more do where a tile's steps would follow one another on a few compute
// units: fp32 products are slow there (32 x 1024 -> 256: 12 us, tiles 50; 300 x 2048 -> 512 38 and 63; 100 x 2048 -> 2048, 2^18 results, 45
// and 43), in 16 bits with long sums alone (64 x 1024 -> 256: 11 us, tiles 15; 64 x 256 -> 256 10 and 9; 32 x 2048 -> 2048, 2^16 results, 18 and 15).
Way way_of(const Call& c)
{
    const long long made = c.P * c.N;
    if (c.P <= kFewRows) return kRowsWay;
    if (is_few(c.dtype, c.K, c.N)) return kStreamWay;
    if (c.dtype == LP_F32 ? c.P <= 512 && made < 1 << 18 : c.P <= 128 && made < 1 << 16 && c.K >= 512) return kRowsWay;
    return is_wide(c, c.N) ? kWideWay : kTileWay;
}
// Its workspace; *n_cu is set where the kernel goes by it.
lp_status forward_bytes(const Call& c, int* n_cu, size_t* bytes)
{
    *bytes = 0;
    const Way way = way_of(c);
    if (way == kWideWay) *bytes = packed_bytes(c.N, c.K);
    if (way != kStreamWay && way != kTileWay) return LP_OK;
    std::string err;
    if (compute_units(n_cu, &err)) return fail(LP_ERR_HIP, err);
    if (way == kTileWay) *bytes = split_of(c, c.K, c.N, *n_cu).bytes;
    return LP_OK;
}

lp_status forward(const lp_linear* q, const void* x, void* y, void* pre, void* workspace, size_t workspace_bytes, hipStream_t s)
{
    Call c;
    lp_status st = validate(q, &c);
    if (st != LP_OK) return st;
    if (c.P == 0) return LP_OK;
    if (!x || !y || !c.weight) return fail(LP_ERR_INVALID_ARG, "x, y and linear->weight must not be NULL");
    if ((st = aligned(c.dtype, {x, y, pre, c.weight, c.residual})) != LP_OK) return st;
    const Way way = way_of(c);
    int n_cu = 0;
    size_t need = 0;
    if ((st = forward_bytes(c, &n_cu, &need)) != LP_OK) return st;
    if (need && (!workspace || workspace_bytes < need))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_linear_workspace_bytes");
    if (need && (uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    LinearDev d;
    std::memset(&d, 0, sizeof(d));
    d.P = c.P; d.K = c.K; d.N = c.N; d.as = c.xs; d.ys = c.ys; d.rs = c.rs;
    d.a = x; d.w = c.weight; d.ws = c.K; d.res = c.residual; d.bias = c.bias; d.out = y; d.keep = pre;
    d.past_cache = bytes_of(c, c.K + (double)c.N * (1 + (pre != nullptr) + (c.residual != nullptr))) > kCacheBytes;
    if (way == kRowsWay) {
        if (c.dtype == LP_BF16) few_rows<__bf16>(d, c.act, s);
        else if (c.dtype == LP_F16) few_rows<_Float16>(d, c.act, s);
        else few_rows<float>(d, c.act, s);
    } else if (way == kWideWay) {
        launch_pack(c.dtype, false, d.w, c.N, c.K, c.K, workspace, s);
        d.w = workspace;
        launch_wide(c.dtype, c.act, false, d, s);
    } else if (way == kStreamWay) {
        launch_stream(c.dtype, c.act, false, d, n_cu, s);
    } else {
        const Split split = split_of(c, c.K, c.N, n_cu);
        d.splits = split.splits;
        d.split_steps = split.steps;
        d.parts = (float*)workspace;
        launch_tiles(c.dtype, c.act, false, d, s);
    }
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
    if (size.all() && (!workspace || workspace_bytes < size.all()))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_linear_workspace_bytes");
    if (size.all() && (uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const Parts p = parts_of(c, n_cu);
    char* at = (char*)workspace;
    float *parts = (float*)(at + size.weight), *bias_parts = (float*)(at + size.weight + size.parts);
    void* dz = size.dz ? at + size.weight + size.parts + size.bias_parts : nullptr;
    const bool params = d_weight || d_bias, skinny = is_skinny(c), halves = c.dtype != LP_F32, join = halves || p.splits > 1;
    const int tiles_k = d_weight ? p.tiles_k : 1;
    if (halves && (params || (skinny && d_x))) {
        BackDev d;
        std::memset(&d, 0, sizeof(d));
        d.P = c.P; d.K = c.K; d.x_channels = d_weight ? c.K : 0; d.N = c.N; d.xs = c.xs; d.ys = c.ys;
        d.x = x; d.dy = d_y; d.pre = pre; d.w = c.weight; d.d_x = skinny ? d_x : nullptr; d.dz = d_x ? dz : nullptr;
        d.parts = parts; d.bias_parts = bias_parts; d.chunk = p.chunk;
        d.tiles_n = p.tiles_n; d.tiles_k = tiles_k; d.splits = p.splits;
        d.d_weight = d_weight != nullptr; d.d_bias = d_bias != nullptr;
        const bool whole = c.K % 8 == 0 && c.N % 8 == 0;
        const auto launch = c.dtype == LP_BF16 ? (whole ? launch_back_bf16_whole : launch_back_bf16_any) : (whole ? launch_back_f16_whole : launch_back_f16_any);
        const hipError_t e = launch(c.act, d, p, skinny, s);
        if (e != hipSuccess) return fail(LP_ERR_HIP, std::string("hipFuncSetAttribute(linear_back_kernel): ") + hipGetErrorString(e));
    } else if (params) {
        WeightDev d;
        std::memset(&d, 0, sizeof(d));
        d.P = c.P; d.K = d_weight ? c.K : 0; d.N = c.N; d.xs = c.xs; d.ys = c.ys;
        d.x = (const float*)x; d.dy = (const float*)d_y; d.pre = (const float*)pre; d.d_weight = d_weight; d.d_bias = d_bias;
        d.parts = join ? parts : nullptr;
        d.bias_parts = join ? bias_parts : nullptr;
        d.chunk = p.chunk; d.tiles_n = p.tiles_n; d.tiles_k = tiles_k; d.splits = p.splits;
        with_act_of(c.act, [&](auto a) {
            const dim3 grid((unsigned)(d.tiles_n * d.tiles_k * p.splits));
            if (p.bn == 64) hipLaunchKernelGGL((linear_weight_kernel<decltype(a)::value, 64>), grid, dim3(kThreads), 0, s, d);
            else hipLaunchKernelGGL((linear_weight_kernel<decltype(a)::value, kWeightTile>), grid, dim3(kThreads), 0, s, d);
        });
    }
    if (params && join) {
        const long long count = (long long)c.N * c.K;
        const JoinDev j = {parts, bias_parts, d_weight, d_bias, count, c.N, p.splits, join_lanes(count, p.splits), join_lanes(c.N, p.splits)};
        const long long each = kThreads / j.lanes * 4, bias_each = kThreads / j.bias_lanes * 4;
        const long long blocks = (d_weight ? (count + each - 1) / each : 0) + (d_bias ? (c.N + bias_each - 1) / bias_each : 0);
        hipLaunchKernelGGL(linear_join_kernel, dim3(grid_of(blocks)), dim3(kThreads), 0, s, j);
    }
    if (d_x && !skinny) {
        LinearDev d;
        std::memset(&d, 0, sizeof(d));
        d.P = c.P; d.K = c.N; d.N = c.K; d.as = c.ys; d.ys = c.xs; d.a = d_y; d.pre = pre; d.w = at; d.out = d_x;
        int act = c.act;
        if (dz && params) {   // d_z is there
            d.a = dz;
            d.as = c.N;
            act = LP_ACT_NONE;
        }
        if (!halves && is_few(c.dtype, c.N, c.K)) {
            d.w = c.weight;
            d.ws = c.K;
            launch_stream(c.dtype, act, true, d, n_cu, s);
        } else if (is_wide(c, c.K) && act == LP_ACT_NONE) {
            launch_pack(c.dtype, true, c.weight, c.K, c.N, c.K, at, s);
            launch_wide(c.dtype, act, true, d, s);
        } else {
            const int chunk = 16 / dtype_bytes(c.dtype);
            d.ws = (c.N + chunk - 1) / chunk * chunk;
            const dim3 grid(grid_of(((c.K + 31ll) / 32) * ((c.N + 31ll) / 32)));
            if (halves) hipLaunchKernelGGL((linear_turn_kernel<uint16_t>), grid, dim3(kThreads), 0, s, (const uint16_t*)c.weight, c.N, c.K, (uint16_t*)at, d.ws);
            else hipLaunchKernelGGL((linear_turn_kernel<float>), grid, dim3(kThreads), 0, s, (const float*)c.weight, c.N, c.K, (float*)at, d.ws);
            const Split split = split_of(c, c.N, c.K, n_cu);
            d.splits = split.splits;
            d.split_steps = split.steps;
            d.parts = (float*)(at + size.all() - size.split);
            launch_tiles(c.dtype, act, true, d, s);
        }
    }
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
    int n_cu = 0;
    if (fwd_bytes) {
        *fwd_bytes = 0;
        const lp_status found = c.P ? lp::forward_bytes(c, &n_cu, fwd_bytes) : LP_OK;
        if (found != LP_OK) return found;
    }
    if (!bwd_bytes) return LP_OK;
    std::string err;
    if (lp::compute_units(&n_cu, &err)) return lp::fail(LP_ERR_HIP, err);
    const lp::Sizes size = lp::sizes(c, n_cu);
    *bwd_bytes = size.all();
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
