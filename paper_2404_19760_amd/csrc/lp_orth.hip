// Orthogonalised updates of weight matrices (Newton-Schulz products) and the optimiser step built on them.
//
//     X_0 = G / (||G||_F + eps),   A = X X^T,   B = a I + b A + c A A,   X <- B X     (X: m x n, m <= n)
//
// Precision: the products magnify what lies in the directions of small singular values (3.44 times a step), so operands of 8
// or 11 bits would leave 1e-3 in the result.  An operand is kept as two fp16 numbers, hi and lo = the rest, at a power-of-two
// scale: 22 bits.  Three matrix products (hi hi + hi lo + lo hi) with fp32 accumulation then have the error of fp32 products
// (measured against 64 bits over five steps: 1e-6 .. 7e-6, 0.7 to 1.14 times that of fp32 torch products) at 16/3 of the fp32 matrix rate.
// fp16 reaches to 65504: the host follows how far singular values can have got in every step (`Plan`) and scales each operand so
// that its bound lies below 2^15; an entry of a matrix is never larger than its largest singular value.
//
// What bounds it: matrix instructions for matrices from some hundreds of rows on, launches below.  X is kept in both orders (X
// and X^T), so that both operands of every product run along memory: A = X X^T from rows of X, A A from rows of A (A is
// symmetric), B X from rows of B and rows of X^T.  A and B are symmetric: only tiles on and above the diagonal are computed,
// and written twice.  a I is added into B, so that B X is all of the step.  Matrices of all lists go through one launch per
// product.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <type_traits>
#include <vector>

#include "lp_kernels.h"
#include "lp_mfma.h"

namespace lp {

namespace {

using half8 = _Float16 __attribute__((ext_vector_type(8)));
using half4 = _Float16 __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kUnits = 256;       // compute units of the chip: what divides the work goes by it
constexpr int kMaxLists = 16;     // lists of one set of launches (their descriptors are the first kernel's arguments)
constexpr int kPad = 64;          // rows and columns of operands are padded to this
constexpr int kNormChunks = 512;  // partial sums of a matrix's norm, at most
constexpr int kChunk = 8192;      // values of one, at least
__host__ __device__ inline int norm_chunks(long long size)
{
    const long long c = (size + kChunk - 1) / kChunk;
    return (int)(c < kNormChunks ? c : kNormChunks);
}

// One list of matrices on the device side.  Layout of a matrix's workspace, in halves from `ws` + i `ws_stride`:
// X and X^T (2 mp np each: hi and lo parts) twice, then A and B (2 mp mp each).
struct List {
    const void* in;     // G of lp_orthogonalize, or the gradients
    void* out;          // the result, or the weights
    float* momentum;    // NULL: lp_orthogonalize
    _Float16* ws;
    long long ws_stride;
    int count, rows, cols;
    int m, n, mp, np;
    int tall;           // rows > cols: X is the transpose
    int dtype;
    float step;         // lr s
    int first_matrix;   // index of its first matrix among all
    int vec4;           // four neighbours can be read and written at a time
    int splits, chunk;  // kPart: parts of the inner dimension, and their steps
    int first_part;     // its first tile's first part among all
};

// How a launch's workgroups are numbered.
struct Launch {
    int total;
    int tiles[kMaxLists];   // of one matrix of a list
    int order[kMaxLists];   // of the products: the longest ones first
    int all[kMaxLists];     // of the products: workgroups of the lists, in the order; else the lists' first ones (behind the last: INT_MAX)
};
enum LaunchOf { kOfNorm, kOfLoad, kOfGram, kOfJoin, kOfPoly, kOfUpdate, kLaunches };

// All that the launches of a call go by.  The first kernel has it as its argument and leaves it in the workspace, where the others
// read it: kernel arguments of 3 KB took the host 7 us a launch.
struct Lists {
    int n, matrices;
    float lr_decay;     // 1 - lr weight_decay
    float mu;
    int nesterov;
    float eps;
    double* norms;      // [matrices][kNormChunks]
    float* parts;       // kPart's tiles, as the waves hold them
    Launch launch[kLaunches];
    List l[kMaxLists];
};
static_assert(sizeof(Lists) % 16 == 0 && sizeof(Lists) <= 3600, "kernel arguments");
using ListsInMemory = const Lists __attribute__((address_space(4)));   // read by scalar loads

__device__ __forceinline__ float load_value(const void* p, size_t i, int dtype)
{
    if (dtype == LP_F32) return ((const float*)p)[i];
    if (dtype == LP_BF16) return (float)((const __bf16*)p)[i];
    return (float)((const _Float16*)p)[i];
}
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// Operands lie in memory in the order in which the matrix instructions take them: blocks of 32 rows x 16 columns, row block by
// row block; of a block first the hi parts, then the lo parts, of each 64 lanes' 16 bytes (lane = row mod 32 + 32 for columns 8 ..
// 15).  A wave loads a block's half with one instruction, to registers or through LDS, both without bank conflicts.
constexpr int kBlock = 1024;   // halves of a block: hi 512, lo 512
// halves from the operand's start to the hi part of element (i, j)
__device__ __forceinline__ size_t at(int i, int j, int width)
{
    return ((size_t)(i >> 5) * (width >> 4) + (j >> 4)) * kBlock + ((i & 31) + ((j & 8) << 2)) * 8 + (j & 7);
}
constexpr int kDepth = 32;   // columns a product takes at a time

using f32x4 = float __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void split4(f32x4 v, half4& hi, half4& lo)
{
    hi = __builtin_convertvector(v, half4);
    lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), half4);
}

// What brings a matrix of this norm to X_0's scale: v -> ldexp(v, e) f (an exponent of its own: no gradient is too large or too small).
struct Scale {
    float f;
    int e;
    __device__ __forceinline__ float operator()(float v) const { return ldexpf(v, e) * f; }
};
__device__ __forceinline__ Scale scale_of(double squares, float eps, float load)
{
    const double norm = sqrt(squares);
    Scale s = {0.0f, 0};
    if (norm != 0.0) s.f = (float)frexp((double)load / (norm + (double)eps), &s.e);
    return s;
}

// The list and the matrix of it that `tile` belongs to, and the tile within the matrix.
template <class L>
__device__ __forceinline__ auto& find(L& a, LaunchOf which, int tile, int& matrix, int& local)
{
    auto& q = a.launch[which];
    int k = 0, from = 0;
#pragma unroll
    for (int i = 1; i < kMaxLists; ++i)
        if (tile >= q.all[i]) {
            k = i;
            from = q.all[i];
        }
    const int tiles = q.tiles[k];
    matrix = (tile - from) / tiles;
    local = tile - from - matrix * tiles;
    return a.l[k];
}

// The same for the products.  Neighbouring workgroups run on different XCDs: each XCD takes a contiguous part of every list's tiles
// (its L2 holds the operands they share; no XCD is left with the long ones), lists in the launch's order.  False: nothing is left.
__device__ __forceinline__ bool find_on_xcd(ListsInMemory& a, LaunchOf which, int block, int& list, int& matrix, int& local)
{
    auto& q = a.launch[which];
    int rest = block >> 3, index = 0;
    list = -1;
#pragma unroll
    for (int k = 0; k < kMaxLists; ++k) {
        const int part = ((block & 7) + 3 * k) & 7;   // (lists of a few tiles do not all fall to the same XCD)
        const int from = q.all[k] * part >> 3, end = q.all[k] * (part + 1) >> 3;   // (at most 2^23 tiles)
        if (list < 0) {
            if (rest < end - from) {
                list = q.order[k];
                index = from + rest;
            }
            rest -= end - from;
        }
    }
    if (list < 0) return false;
    const int tiles = q.tiles[list];
    matrix = index / tiles;
    local = index - matrix * tiles;
    return true;
}

// Four neighbouring values from `i` on, of which `left` are there.
__device__ __forceinline__ f32x4 load4(const void* p, size_t i, int dtype, bool vec4, int left)
{
    f32x4 v = {};
    if (vec4) {
        if (dtype == LP_F32) return *(const f32x4*)((const float*)p + i);
        if (dtype == LP_BF16) {
            using b4 = __bf16 __attribute__((ext_vector_type(4)));
            const b4 q = *(const b4*)((const __bf16*)p + i);
            for (int e = 0; e < 4; ++e) v[e] = (float)q[e];
        } else {
            const half4 q = *(const half4*)((const _Float16*)p + i);
            for (int e = 0; e < 4; ++e) v[e] = (float)q[e];
        }
        return v;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) v[e] = load_value(p, i + e, dtype);
    return v;
}

// Sums of squares in 64 bits (so that no gradient is too large or too small), one workgroup a (matrix, chunk); the optimiser
// step updates the momentum on the way.
__global__ __launch_bounds__(kThreads) void orth_norm_kernel(Lists a, Lists* in_memory)
{
    if (blockIdx.x == 0) {   // (the lists are the first argument: taken by address they would be copied to scratch memory)
        const auto* from = (const uint32_t __attribute__((address_space(4)))*)__builtin_amdgcn_kernarg_segment_ptr();
        for (int i = threadIdx.x; i < (int)(sizeof(Lists) / 4); i += kThreads) ((uint32_t*)in_memory)[i] = from[i];
    }
    __shared__ double lds[4];
    int matrix, chunk;
    const List& l = find(a, kOfNorm, blockIdx.x, matrix, chunk);
    const int chunks = norm_chunks((long long)l.rows * l.cols);
    const long long size = (long long)l.rows * l.cols, from = (long long)matrix * size;
    double sum = 0.0;
    for (long long i = ((long long)chunk * kThreads + threadIdx.x) * 4; i < size; i += (long long)chunks * kThreads * 4) {
        const int left = (int)min(size - i, 4ll);
        f32x4 v = load4(l.in, from + i, l.dtype, l.vec4, left);
        if (l.momentum) {
            const f32x4 m = load4(l.momentum, from + i, LP_F32, l.vec4, left);
            f32x4 to;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                to[e] = fmaf(a.mu, m[e], v[e]);
                v[e] = a.nesterov ? fmaf(a.mu, to[e], v[e]) : to[e];
            }
            if (l.vec4) {
                *(f32x4*)(l.momentum + from + i) = to;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) l.momentum[from + i + e] = to[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) sum += (double)v[e] * (double)v[e];
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.norms[(size_t)(l.first_matrix + matrix) * kNormChunks + chunk] = lds[0] + lds[1] + lds[2] + lds[3];
}

// X_0 and its transpose as operands, padded with zeros: one workgroup a 64 x 64 tile of G.
__global__ __launch_bounds__(kThreads) void orth_load_kernel(const Lists* lists, float scale)
{
    ListsInMemory& a = *(ListsInMemory*)lists;
    __shared__ float tile[64 * 65];
    __shared__ double sums[4];
    int matrix, local;
    auto& l = find(a, kOfLoad, blockIdx.x, matrix, local);
    const long long size = (long long)l.rows * l.cols;
    const int chunks = norm_chunks(size);
    double norm = 0.0;
    for (int i = threadIdx.x; i < chunks; i += kThreads) norm += a.norms[(size_t)(l.first_matrix + matrix) * kNormChunks + i];
    for (int o = 32; o; o >>= 1) norm += __shfl_xor(norm, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = norm;
    const int rp = l.tall ? l.np : l.mp, cp = l.tall ? l.mp : l.np;   // padded rows and columns of G
    const int tr = local / (cp / 64), tc = local - tr * (cp / 64);
    const long long from = (long long)matrix * size;
    const int c4 = (threadIdx.x & 15) * 4;
    f32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int gr = tr * 64 + (threadIdx.x >> 4) + 16 * k, gc = tc * 64 + c4;
        v[k] = f32x4{};
        if (gr < l.rows && gc < l.cols) {
            const size_t i = from + (size_t)gr * l.cols + gc;
            const int left = min(l.cols - gc, 4);
            const bool vec4 = l.vec4 && left == 4 && (l.cols & 3) == 0;
            v[k] = load4(l.in, i, l.dtype, vec4, left);
            if (l.momentum) {
                const f32x4 m = load4(l.momentum, i, LP_F32, vec4, left);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k][e] = a.nesterov ? fmaf(a.mu, m[e], v[k][e]) : m[e];
            }
        }
    }
    __syncthreads();
    const Scale f = scale_of(sums[0] + sums[1] + sums[2] + sums[3], a.eps, scale);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[((threadIdx.x >> 4) + 16 * k) * 65 + c4 + e] = f(v[k][e]);
    __syncthreads();
    _Float16* ws = l.ws + (size_t)matrix * l.ws_stride;
    const size_t plane = (size_t)2 * l.mp * l.np;
    _Float16* same = ws + (l.tall ? plane : 0);    // the operand in the order of G
    _Float16* other = ws + (l.tall ? 0 : plane);   // its transpose
    // a lane's 16 bytes: row r of a block of 32, columns c .. c + 7
    const int lane = threadIdx.x & 63, r = lane & 31, c = (threadIdx.x >> 6) * 16 + (lane >> 5) * 8;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        half8 hi, lo, thi, tlo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 vh, vl;
            split(tile[(k * 32 + r) * 65 + c + e], vh, vl);
            hi[e] = vh; lo[e] = vl;
            split(tile[(c + e) * 65 + k * 32 + r], vh, vl);
            thi[e] = vh; tlo[e] = vl;
        }
        _Float16* to = same + at(tr * 64 + k * 32 + r, tc * 64 + c, cp);
        *(half8*)to = hi;
        *(half8*)(to + 512) = lo;
        to = other + at(tc * 64 + k * 32 + r, tr * 64 + c, rp);
        *(half8*)to = thi;
        *(half8*)(to + 512) = tlo;
    }
}

enum Product { kGram, kPoly, kUpdate, kLast, kPart, kJoin };   // kPart: a part of kGram's inner dimension; kJoin adds the parts

// Scales of one step: what the accumulator is multiplied with, and the polynomial's coefficients at B's scale.
struct Step {
    float acc;          // kGram, kUpdate: scale of the result over the operands'; kLast: 1 over the operands'; kPoly: c's factor
    float diag, lin;    // kPoly: a and b at B's scale
    int from, to;       // which of the two X's is read, written
};

using GlobalPtr = __attribute__((address_space(1))) const void;
using LdsPtr = __attribute__((address_space(3))) void;

// One workgroup of eight waves a TILE x TILE tile of P Q^T.  A wave has all rows and 32 columns of the tile, so TILE / 32 waves
// make a group that covers it, and the groups share the inner dimension among themselves; at the end they exchange sums through LDS,
// and each finishes a part of the rows.  So a compute unit with a single tile has two waves on every SIMD.
//
// The loop's step is 32 columns of P and Q.  P goes through LDS (two buffers in turn), Q, of which no two waves of a group need the
// same, straight to registers.  For 128 x 128 this keeps both ways below the matrix cores' time: of 768 cycles for a group's step
// LDS (128 bytes a cycle) takes 640, the cache (64 bytes a cycle) 512.  With waves of 64 x 64 and both operands in LDS it would be
// 768 and 512, with Q in registers 384 and 768.  A row block's registers are read again, for the next half step, as soon as they
// have been used, and the workgroup meets in the middle of a step, so that a wave always has products to issue behind the barrier.
// The small products (hi lo + lo hi) have an accumulator of their own: added into the large one's they would round it three
// times as often (error against 64 bits at 2048 x 2048: 6.8e-6 in one accumulator, 4.4e-6 in two; fp32 torch 4.2e-6).
// Measured on 2 x 2048 x 2048 and 1024 x 4096: B X 129 us (1.0 PFLOP/s of fp16 products; a library product of 8192^3 1.08), A = X X^T
// 94 to 105, A A 87 (308 tiles on 256 units); on 36 matrices of width 512 88, 62 and 39 us.
template <int TILE, int GROUPS>
struct ProductShape {
    static constexpr int kWaves = TILE / 32, kGroups = GROUPS, kGroupThreads = 64 * kWaves;
    static constexpr int kThreadsOf = kGroups * kGroupThreads;
    static constexpr int kBuffer = TILE * kDepth * 4;         // bytes of a step's P
    static constexpr int kValues = TILE / 2;                  // sums of a lane: TILE / 32 blocks of 16
    static constexpr int kMine = kValues / kGroups;           // of them a group finishes
    static constexpr int kBuffers = kGroups * 2 * kBuffer, kExchange = kGroups * (kGroups - 1) * kWaves * kMine * 64 * 4, kTurn = kGroups * kWaves * 32 * 33 * 4;
    static constexpr int kLds = kBuffers > kExchange ? (kBuffers > kTurn ? kBuffers : kTurn) : (kExchange > kTurn ? kExchange : kTurn);
};

template <Product WHAT, int TILE, int GROUPS>
__global__ __launch_bounds__((ProductShape<TILE, GROUPS>::kThreadsOf), (2)) void orth_product_kernel(const Lists* lists, Step s)
{
    ListsInMemory& a = *(ListsInMemory*)lists;
    using S = ProductShape<TILE, GROUPS>;
    constexpr int F = TILE / 32;                    // row blocks
    constexpr int kLoads = S::kBuffer / (S::kGroupThreads * 16);
    __shared__ alignas(16) char lds[S::kLds];
    int list = 0, matrix = 0, local = 0;
    constexpr LaunchOf kWhich = WHAT == kGram || WHAT == kPart ? kOfGram : WHAT == kJoin ? kOfJoin : WHAT == kPoly ? kOfPoly : kOfUpdate;
    if (!find_on_xcd(a, kWhich, blockIdx.x, list, matrix, local)) return;
    auto& l = a.l[list];
    _Float16* ws = l.ws + (size_t)matrix * l.ws_stride;
    const size_t plane = (size_t)2 * l.mp * l.np, square = (size_t)2 * l.mp * l.mp;
    _Float16* x = ws + s.from * 2 * plane;
    _Float16* A = ws + 4 * plane;
    _Float16* B = A + square;
    constexpr bool kGramLike = WHAT == kGram || WHAT == kPart || WHAT == kJoin, kSymmetric = kGramLike || WHAT == kPoly;
    int ti, tj, slice = 0;
    const int mt = (l.mp + TILE - 1) / TILE, nt = (l.np + TILE - 1) / TILE;
    const int part = l.first_part + (matrix * a.launch[kWhich].tiles[list] + local) * (WHAT == kJoin ? l.splits : 1);
    if (WHAT == kPart) {
        slice = local % l.splits;
        local /= l.splits;
    }
    if (kSymmetric) {   // tiles on and above the diagonal, row by row
        ti = 0;
        int rest = local;
        while (rest >= mt - ti) rest -= mt - ti++;
        tj = ti + rest;
    } else {
        ti = local / nt;
        tj = local - ti * nt;
    }
    const _Float16* p = kGramLike ? x : WHAT == kPoly ? A : B;
    const _Float16* q = kGramLike ? x : WHAT == kPoly ? A : x + plane;
    const int K = kGramLike ? l.np : l.mp;
    const int p_blocks = l.mp >> 5, q_blocks = (kSymmetric ? l.mp : l.np) >> 5;
    const int wave_of_8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave_of_8 / S::kWaves, wave = wave_of_8 % S::kWaves;
    const int lane = threadIdx.x & 63, in_group = threadIdx.x % S::kGroupThreads, l32 = lane & 31, h = lane >> 5;
    float mine[S::kMine];   // what this wave finishes
    auto part_at = [&](int k, int e) { return (f32x4*)(a.parts + (size_t)k * TILE * TILE) + wave_of_8 * (S::kMine * 16) + (e >> 2) * 64 + lane; };
    if constexpr (WHAT == kJoin) {
#pragma unroll
        for (int e = 0; e < S::kMine; ++e) mine[e] = 0.0f;
        for (int k = 0; k < l.splits; ++k)
#pragma unroll
            for (int e = 0; e < S::kMine; e += 4) {
                const f32x4 v = *part_at(part + k, e);
#pragma unroll
                for (int j = 0; j < 4; ++j) mine[e + j] += v[j];
            }
    } else {
    // a group's steps; where they do not divide evenly the last ones have fewer
    const int begin = WHAT == kPart ? slice * l.chunk : 0, all = WHAT == kPart ? min(K / kDepth, begin + l.chunk) : K / kDepth;
    const int steps = (all - begin + S::kGroups - 1) / S::kGroups, start = begin + group * steps, mine_steps = min(steps, all - start);
    // row blocks behind an operand's end are its last one again (their products are not stored)
    const size_t row = (size_t)(K >> 4) * kBlock;   // halves of a row block
    const _Float16 *p_at[kLoads], *q_at;            // the same for all lanes
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        const int at_byte = u * S::kGroupThreads * 16;   // of the step's P: 4096 of every row block
        p_at[u] = p + min(ti * F + at_byte / 4096, p_blocks - 1) * row + at_byte % 4096 / 2;
    }
    q_at = q + min(tj * F + wave, q_blocks - 1) * row;
    char* buffers = lds + group * 2 * S::kBuffer;
    half8 staged[2][kLoads];   // P of two steps
    half8 qv[4][2];   // Q of two steps: 16-column half of a step, hi or lo
    auto ask_p = [&](int step, half8 (&v)[kLoads]) {
        step = min(start + step, all - 1);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) v[u] = *(const half8*)(p_at[u] + (size_t)step * (2 * kBlock) + in_group * 8);
    };
    auto put_p = [&](int buffer, bool any, const half8 (&v)[kLoads]) {
        char* to = buffers + buffer * S::kBuffer + in_group * 16;
        if (any) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) *(half8*)(to + u * S::kGroupThreads * 16) = v[u];
        } else {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) *(half8*)(to + u * S::kGroupThreads * 16) = half8{};
        }
    };
    auto ask_q = [&](int k, half8 (&to)[2]) {   // k: half steps
        k = min(2 * start + k, 2 * all - 1);
#pragma unroll
        for (int c = 0; c < 2; ++c) to[c] = *(const half8*)(q_at + (size_t)k * kBlock + c * 512 + lane * 8);
    };
    half8 pv[F][2];
    auto get_p = [&](int buffer, int k, int f) {
#pragma unroll
        for (int c = 0; c < 2; ++c) pv[f][c] = *(const half8*)(buffers + buffer * S::kBuffer + f * 4096 + (2 * k + c) * 1024 + lane * 16);
    };
    f32x16 acc[F] = {}, cross[F] = {};
    ask_p(0, staged[0]);
#pragma unroll
    for (int k = 0; k < 4; ++k) ask_q(k, qv[k]);
    put_p(0, mine_steps > 0, staged[0]);
    ask_p(1, staged[1]);
    ask_p(2, staged[0]);
    __syncthreads();
#pragma unroll
    for (int f = 0; f < F; ++f) get_p(0, 0, f);
    for (int first = 0; first < steps; first += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int step = first + u;
            put_p(u ^ 1, step + 1 < mine_steps, staged[u ^ 1]);   // (behind the last step P is zero: what is left of the loop adds nothing)
            ask_p(step + 3, staged[u ^ 1]);
            __builtin_amdgcn_sched_barrier(0);     // (everything is asked for and used in the order written)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                half8 (&q2)[2] = qv[2 * u + k];
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    cross[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pv[i][1], q2[0], cross[i], 0, 0, 0);
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pv[i][0], q2[0], acc[i], 0, 0, 0);
                    cross[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pv[i][0], q2[1], cross[i], 0, 0, 0);
                    // the same rows of the next half step: they arrive while the other rows are multiplied
                    get_p(k ? u ^ 1 : u, k ^ 1, i);
                    __builtin_amdgcn_sched_barrier(0);
                }
                ask_q(2 * step + k + 4, q2);
                __builtin_amdgcn_sched_barrier(0);
                // in the middle of a step: the next step's P is there, and nobody reads this step's any more
                if (k == 0) __syncthreads();
            }
        }
    }
    __syncthreads();
    // group g finishes values g kMine .. of every lane; the groups' sums are added in their order
    if constexpr (S::kGroups == 1) {
#pragma unroll
        for (int e = 0; e < S::kMine; ++e) mine[e] = acc[e >> 4][e & 15] + cross[e >> 4][e & 15];
    } else {
        auto slot = [&](int to, int from, int e) {
            return (f32x4*)lds + ((to * (S::kGroups - 1) + from - (from > to)) * S::kWaves + wave) * (S::kMine * 16) + (e >> 2) * 64 + lane;
        };
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
            for (int e = 0; e < S::kMine; e += 4) {
                f32x4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at_value = g * S::kMine + e + j;
                    v[j] = acc[at_value >> 4][at_value & 15] + cross[at_value >> 4][at_value & 15];
                }
                if (g == group) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) mine[e + j] = v[j];
                } else {
                    *slot(g, group, e) = v;
                }
            }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < S::kMine; e += 4) {
            f32x4 v = {};
#pragma unroll
            for (int g = 0; g < S::kGroups; ++g) {
                const f32x4 own = {mine[e], mine[e + 1], mine[e + 2], mine[e + 3]};
                v += g == group ? own : *slot(group, g, e);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) mine[e + j] = v[j];
        }
        __syncthreads();
    }
    if (WHAT == kPart) {
#pragma unroll
        for (int e = 0; e < S::kMine; e += 4) *part_at(part, e) = f32x4{mine[e], mine[e + 1], mine[e + 2], mine[e + 3]};
        return;
    }
    }
    // value e of a lane: row 8 (e / 4) + 4 h + e % 4, column l32 of a 32 x 32 block.  Four rows of a column are neighbours in an
    // operand whose rows are the block's columns; for the other order the rows are turned over in the wave's own LDS.
    constexpr int kRows = S::kMine >= 16 ? 32 : 16;   // rows of a block that this wave finishes
    constexpr int kFinish = S::kMine >= 16 ? S::kMine / 16 : 1;
    uint32_t* turn = (uint32_t*)lds + wave_of_8 * (32 * 33);
    const int jb = tj * TILE + wave * 32;
    if constexpr (WHAT == kLast) {
        // Row by row of G's order: of a tall G neighbouring lanes take neighbouring block rows.  Value e of a lane lies dr(e) rows
        // behind its first one.  All weights are read before the first is written: a read behind a write would wait for it.
        constexpr int kOut = kRows / 2;
        auto dr = [&](int e) { return l.tall ? e * (64 / kRows) : 8 * (e >> 2) + (e & 3); };
        auto first_row = [&](int ib) { return l.tall ? jb + lane / kRows : ib + 4 * h; };
        auto column = [&](int ib) { return l.tall ? ib + (lane & (kRows - 1)) : jb + l32; };
        auto place = [&](int ib) { return ((size_t)matrix * l.rows + first_row(ib)) * l.cols + column(ib); };
        float old[kFinish][kOut];
        if (l.momentum) {
#pragma unroll
            for (int fi = 0; fi < kFinish; ++fi) {
                const int ib = ti * TILE + (group * kFinish + fi) * kRows;
                const float* w = (const float*)l.out + place(ib);
                const int r = first_row(ib);
                const bool in = column(ib) < l.cols;
#pragma unroll
                for (int e = 0; e < kOut; ++e)
                    if (in && r + dr(e) < l.rows) old[fi][e] = w[(size_t)dr(e) * l.cols];
            }
        }
#pragma unroll
        for (int fi = 0; fi < kFinish; ++fi) {
            const int ib = ti * TILE + (group * kFinish + fi) * kRows;
            if ((ib >> 5) >= p_blocks || (jb >> 5) >= q_blocks) continue;
            float v[kOut];
#pragma unroll
            for (int e = 0; e < kOut; ++e) v[e] = mine[fi * 16 + e] * s.acc;
            if (l.tall) {
#pragma unroll
                for (int e = 0; e < kOut; ++e) turn[(8 * (e >> 2) + 4 * h + (e & 3)) * 33 + l32] = __float_as_uint(v[e]);
                wave_lds_fence();
#pragma unroll
                for (int e = 0; e < kOut; ++e) v[e] = __uint_as_float(turn[(lane & (kRows - 1)) * 33 + e * (64 / kRows) + lane / kRows]);
                wave_lds_fence();
            }
            const size_t at_first = place(ib);
            const int r = first_row(ib);
            const bool in = column(ib) < l.cols;
            auto each = [&](auto&& f) {
#pragma unroll
                for (int e = 0; e < kOut; ++e)
                    if (in && r + dr(e) < l.rows) f(e, (size_t)dr(e) * l.cols);
            };
            if (l.momentum) {
                float* w = (float*)l.out + at_first;
                each([&](int e, size_t i) { w[i] = fmaf(-l.step, v[e], a.lr_decay * old[fi][e]); });
            } else if (l.dtype == LP_F32) {
                float* to = (float*)l.out + at_first;
                each([&](int e, size_t i) { to[i] = v[e]; });
            } else if (l.dtype == LP_BF16) {
                __bf16* to = (__bf16*)l.out + at_first;
                each([&](int e, size_t i) { to[i] = (__bf16)v[e]; });
            } else {
                _Float16* to = (_Float16*)l.out + at_first;
                each([&](int e, size_t i) { to[i] = (_Float16)v[e]; });
            }
        }
        return;
    }
#pragma unroll
    for (int fi = 0; fi < kFinish; ++fi) {
        const int ib = ti * TILE + (group * kFinish + fi) * kRows;
        if ((ib >> 5) >= p_blocks || (jb >> 5) >= q_blocks) continue;
        _Float16* direct = kGramLike ? A : WHAT == kPoly ? B : ws + s.to * 2 * plane;
        _Float16* trans = WHAT == kUpdate ? direct + plane : direct;
        const int width = WHAT == kUpdate ? l.np : l.mp;
        const bool both = WHAT == kUpdate || ti != tj;   // (a tile on the diagonal is its own transpose)
#pragma unroll
        for (int e4 = 0; e4 < kRows / 8; ++e4) {
            half4 hi, lo, ah, al;
            const int r = 8 * e4 + 4 * h;
            const size_t to = at(jb + l32, ib + r, l.mp);
            if (WHAT == kPoly) {
                ah = *(const half4*)(A + to);
                al = *(const half4*)(A + to + 512);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v = mine[fi * 16 + 4 * e4 + e] * s.acc;
                if (WHAT == kPoly) {
                    v = fmaf(s.lin, (float)ah[e] + (float)al[e], v);
                    if (ib + r + e == jb + l32 && jb + l32 < l.m) v += s.diag;
                }
                _Float16 vh, vl;
                split(v, vh, vl);
                hi[e] = vh;
                lo[e] = vl;
                if (both) turn[(r + e) * 33 + l32] = (uint32_t)__builtin_bit_cast(uint16_t, vh) | (uint32_t)__builtin_bit_cast(uint16_t, vl) << 16;
            }
            *(half4*)(trans + to) = hi;
            *(half4*)(trans + to + 512) = lo;
        }
        if (both) {
            wave_lds_fence();
#pragma unroll
            for (int k = 0; k < kRows / 16; ++k) {
                const int r = lane & (kRows - 1), c = k * 16 + lane / kRows * 8;
                half8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t v = turn[r * 33 + c + e];
                    hi[e] = __builtin_bit_cast(_Float16, (uint16_t)v);
                    lo[e] = __builtin_bit_cast(_Float16, (uint16_t)(v >> 16));
                }
                _Float16* to = direct + at(ib + r, jb + c, width);
                *(half8*)to = hi;
                *(half8*)(to + 512) = lo;
            }
            wave_lds_fence();
        }
    }
}

// Scales of all steps from the bounds of what the operands can hold.
struct Plan {
    float load;   // of X_0
    Step gram[LP_ORTH_MAX_STEPS], poly[LP_ORTH_MAX_STEPS], update[LP_ORTH_MAX_STEPS];
    int steps;
};

// ---- small matrices: a workgroup does all of it --------------------------------------------------------------------

// Matrices of at most 64 x 128 (a decoder's layers): one workgroup of four waves keeps X, X^T, A and B in LDS, in the same order as
// the large operands, from the gradient to the result: one launch, and no bytes but G's and the result's (the optimiser's: the
// momentum's and the weights').  Its time is that of a chain of 3 x steps products with a barrier behind each: 64 x 64 in 2.1 us a
// step and 10 us before and after them (in the launches of the large matrices: 86 us for the three matrices of a decoder, here 20.7).
// Rows and columns are padded to 32.  A wave has one 32 x 32 block of A and B and up to two of X.
constexpr int kSmallM = 64, kSmallN = 128;
// Longer ones as far as X and X^T fit the LDS: 64 x 224 and 32 x 448 (in the launches of the large
// ones 101 us for 64 x 224, 109 for 30 x 448, 118 for 31 of 20 x 400; here 41, 43 and 41).  Their columns are padded to sizes that the steps are built for.
__host__ __device__ inline int pad32(int v) { return (v + 31) & ~31; }
__host__ __device__ inline int small_columns(int mp, int n) { return n <= kSmallN ? pad32(n) : mp == 64 ? (n <= 192 ? 192 : 224) : (n + 63) & ~63; }
__host__ __device__ inline bool fits_one_workgroup(int rows, int cols)
{
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return m <= kSmallM && n <= (m <= 32 ? 448 : 224);
}
// LDS: X, X^T, B, then A (the waves' blocks to turn over lie over it); G in 32 bits lies over all but X before they are made.
__host__ __device__ inline int small_lds(int mp, int np)
{
    const int turn = 4 * 32 * 33 * 4, square = mp * mp * 4, g = mp * (np + 1) * 4;
    const int rest = mp * np * 4 + square + (square > turn ? square : turn);
    return mp * np * 4 + (rest > g ? rest : g);
}
constexpr int kSmallLds = 64 * 224 * 8 + 64 * 64 * 4 + 4 * 32 * 33 * 4;   // of 64 x 224, the most

// The lists of such matrices, and what the steps go by (all that this kernel is given: 1.4 KB).
struct SmallList {
    const void* in;
    void* out;
    float* momentum;
    int rows, cols, m, n, tall, dtype, vec4;
    float step;
};
struct SmallCall {
    int n, nesterov;
    float lr_decay, mu, eps, load;
    int steps;
    int first[kMaxLists];            // workgroups, as in Launch
    SmallList l[kMaxLists];
    float v[LP_ORTH_MAX_STEPS][5];   // scales of a step: kGram's, kPoly's three, kUpdate's
};

// Block (bi, bj) of P Q^T over 16 K16 columns.
template <int K16>
__device__ __forceinline__ f32x16 small_product(const _Float16* p, const _Float16* q, int bi, int bj)
{
    const int lane = threadIdx.x & 63;
    f32x16 acc = {}, cross = {};
    const _Float16* pb = p + bi * K16 * kBlock + lane * 8;
    const _Float16* qb = q + bj * K16 * kBlock + lane * 8;
#pragma unroll
    for (int k = 0; k < K16; ++k) {
        const half8 ph = *(const half8*)(pb + k * kBlock), pl = *(const half8*)(pb + k * kBlock + 512);
        const half8 qh = *(const half8*)(qb + k * kBlock), ql = *(const half8*)(qb + k * kBlock + 512);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
        cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, cross, 0, 0, 0);
        cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, cross, 0, 0, 0);
    }
    return acc + cross;
}

// The steps of a matrix of MB x NB blocks of 32 x 32 (sizes are constants: at one wave a SIMD every index that is worked out
// between two barriers is waited for), and the result.
template <int MB, int NB>
__device__ __forceinline__ void small_steps(const SmallCall& a, const SmallList& l, int n_steps, const float* scales, _Float16* X, _Float16* XT,
                                            _Float16* B, _Float16* A, const float* g, const Scale& f, size_t from)
{
    constexpr int kPer = (MB * NB + 3) / 4;   // blocks of X that a wave has, at most
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    uint32_t* turn = (uint32_t*)A + wave * (32 * 33);
    const int bi = wave >> 1, bj = wave & 1;   // of A and B
    const bool square = bi < MB && bj < MB;
    int xi[kPer], xj[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        xi[u] = (wave + 4 * u) / NB;
        xj[u] = (wave + 4 * u) % NB;
    }
    // block (bi, bj) as block (bj, bi) of an operand of 32 W columns: a lane's four rows are neighbours there
    auto put_turned = [&](const half4 (&hi)[4], const half4 (&lo)[4], _Float16* to, int W, int rb, int cb) {
        _Float16* dst = to + (cb * 2 * W + rb * 2) * kBlock + l32 * 8 + 4 * h;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {   // rows 8 e4 + 4 h ..: block e4 / 2, its half e4 % 2
            *(half4*)(dst + (e4 >> 1) * kBlock + (e4 & 1) * 256) = hi[e4];
            *(half4*)(dst + (e4 >> 1) * kBlock + (e4 & 1) * 256 + 512) = lo[e4];
        }
    };
    auto split16 = [&](const f32x16& v, half4 (&hi)[4], half4 (&lo)[4]) {
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) split4(f32x4{v[4 * e4], v[4 * e4 + 1], v[4 * e4 + 2], v[4 * e4 + 3]}, hi[e4], lo[e4]);
    };
    // blocks of X, one a wave at a time: the 16 bytes of a lane are row i, columns j .. of the operand
    constexpr int kBlocks = MB * NB * 2, kRow = NB * 32 + 1;
#pragma unroll 2
    for (int block = wave; block < kBlocks; block += 4) {
        const float* src = g + (block / (2 * NB) * 32 + l32) * kRow + block % (2 * NB) * 16 + 8 * h;
        _Float16* to = X + block * kBlock + lane * 8;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            half4 wh, wl;
            split4(f32x4{f(src[4 * q]), f(src[4 * q + 1]), f(src[4 * q + 2]), f(src[4 * q + 3])}, wh, wl);
            *(half4*)(to + 4 * q) = wh;
            *(half4*)(to + 512 + 4 * q) = wl;
        }
    }
    __syncthreads();   // (X^T lies where G was)
#pragma unroll 2
    for (int block = wave; block < kBlocks; block += 4) {
        // row j of X^T, columns i .. i + 7: column j of X, whose rows lie 16 bytes apart
        const int j = block / (2 * MB) * 32 + l32, i = block % (2 * MB) * 16 + 8 * h;
        const _Float16* src = X + ((i >> 5) * 2 * NB + (j >> 4)) * kBlock + ((i & 31) + ((j & 8) << 2)) * 8 + (j & 7);
        half8 wh, wl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            wh[e] = src[e * 8];
            wl[e] = src[e * 8 + 512];
        }
        *(half8*)(XT + block * kBlock + lane * 8) = wh;
        *(half8*)(XT + block * kBlock + 512 + lane * 8) = wl;
    }
    float diagonal[16];   // 1 on it
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int i = bi * 32 + 8 * (e >> 2) + 4 * h + (e & 3), j = bj * 32 + l32;
        diagonal[e] = i == j && i < l.m ? 1.0f : 0.0f;
    }
    __syncthreads();
    half4 hi[4], lo[4];
#pragma unroll 1
    for (int step = 0; step < n_steps; ++step) {
        const float s_gram = scales[5 * step], s_poly = scales[5 * step + 1], s_diag = scales[5 * step + 2], s_lin = scales[5 * step + 3],
                    s_update = scales[5 * step + 4];
        f32x16 gram = {};
        if (square) {
            gram = small_product<2 * NB>(X, X, bi, bj) * s_gram;
            split16(gram, hi, lo);
            put_turned(hi, lo, A, MB, bi, bj);
        }
        __syncthreads();
        if (square) {
            f32x16 v = small_product<2 * MB>(A, A, bi, bj);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = fmaf(s_diag, diagonal[e], fmaf(s_lin, gram[e], v[e] * s_poly));
            split16(v, hi, lo);
            put_turned(hi, lo, B, MB, bi, bj);
        }
        __syncthreads();
        if (step + 1 < n_steps) {
            f32x16 next[kPer];
#pragma unroll
            for (int u = 0; u < kPer; ++u)
                if (wave + 4 * u < MB * NB) next[u] = small_product<2 * MB>(B, XT, xi[u], xj[u]) * s_update;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                if (wave + 4 * u >= MB * NB) continue;
                split16(next[u], hi, lo);
                put_turned(hi, lo, XT, MB, xi[u], xj[u]);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    turn[(8 * (e >> 2) + 4 * h + (e & 3)) * 33 + l32] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi[e >> 2][e & 3]) |
                                                                        (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo[e >> 2][e & 3]) << 16;
                wave_lds_fence();
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    half8 rh, rl;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t v = turn[l32 * 33 + k * 16 + h * 8 + e];
                        rh[e] = __builtin_bit_cast(_Float16, (uint16_t)v);
                        rl[e] = __builtin_bit_cast(_Float16, (uint16_t)(v >> 16));
                    }
                    _Float16* dst = X + (xi[u] * 2 * NB + xj[u] * 2 + k) * kBlock + lane * 8;
                    *(half8*)dst = rh;
                    *(half8*)(dst + 512) = rl;
                }
                wave_lds_fence();
            }
            __syncthreads();
        } else {
            // the result in G's order: of a tall G the transposed product, so that neighbouring lanes have neighbouring columns
            const _Float16 *p = l.tall ? XT : B, *q = l.tall ? B : XT;
#pragma unroll 1
            for (int u = wave; u < MB * NB; u += 4) {
                const int x0 = u / NB, x1 = u % NB, ri = l.tall ? x1 : x0, ci = l.tall ? x0 : x1, rb = ri * 32, c = ci * 32 + l32;
                const f32x16 v = small_product<2 * MB>(p, q, ri, ci) * s_update;
                auto each = [&](auto&& f) {   // (offsets from the matrix's start: 32 bits)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int r = rb + 8 * (e >> 2) + 4 * h + (e & 3);
                        if (r < l.rows && c < l.cols) f(e, (unsigned)(r * l.cols + c));
                    }
                };
                if (l.momentum) {
                    float* to = (float*)l.out + from;
                    float w[16];
                    each([&](int e, unsigned i) { w[e] = to[i]; });
                    each([&](int e, unsigned i) { to[i] = fmaf(-l.step, v[e], a.lr_decay * w[e]); });
                } else if (l.dtype == LP_F32) {
                    float* to = (float*)l.out + from;
                    each([&](int e, unsigned i) { to[i] = v[e]; });
                } else if (l.dtype == LP_BF16) {
                    __bf16* to = (__bf16*)l.out + from;
                    each([&](int e, unsigned i) { to[i] = (__bf16)v[e]; });
                } else {
                    _Float16* to = (_Float16*)l.out + from;
                    each([&](int e, unsigned i) { to[i] = (_Float16)v[e]; });
                }
            }
        }
    }
}

template <bool LONG>
__global__ __launch_bounds__(kThreads) void orth_small_kernel(SmallCall a)
{
    extern __shared__ char small_bytes[];
    __shared__ double sums[4];
    __shared__ float scales[LP_ORTH_MAX_STEPS * 5];   // (read once: as arguments every step's would wait for a line of its own)
    const float my_scale = threadIdx.x < LP_ORTH_MAX_STEPS * 5 ? a.v[threadIdx.x / 5][threadIdx.x % 5] : 0.0f;   // (stored once G is asked for)
    int list = 0, matrix = blockIdx.x;
#pragma unroll
    for (int i = 1; i < kMaxLists; ++i)
        if ((int)blockIdx.x >= a.first[i]) {
            list = i;
            matrix = (int)blockIdx.x - a.first[i];
        }
    const SmallList& l = a.l[list];
    const int m = l.m, n = l.n, mp = pad32(m), np = small_columns(mp, n);
    _Float16* X = (_Float16*)small_bytes;
    _Float16* XT = X + 2 * mp * np;
    _Float16* B = XT + 2 * mp * np;
    _Float16* A = B + 2 * mp * mp;
    float* g = (float*)XT;   // [mp][np + 1], X's order
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const size_t from = (size_t)matrix * l.rows * l.cols;
    // G: a thread has four columns of every kPasses-th group of rows
    constexpr int kPasses = LONG ? 16 : 8;   // 32 x 448 in rows of 128 lanes, 64 x 224 in rows of 64; 64 x 128 in rows of 32
    const int shift = l.cols > 256 ? 7 : l.cols > 128 ? 6 : l.cols > 64 ? 5 : l.cols > 32 ? 4 : 3;
    const int c0 = (threadIdx.x & ((1 << shift) - 1)) * 4, r0 = threadIdx.x >> shift, dr = kThreads >> shift;
    const int left = l.cols - c0;
    const bool vec4 = l.vec4 && (l.cols & 3) == 0;
    f32x4 v[kPasses], mom[kPasses];
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
        const int r = r0 + k * dr;
        const bool in = r < l.rows && left > 0;
        v[k] = in && l.dtype == LP_F32 ? load4(l.in, from + r * l.cols + c0, LP_F32, vec4, left) : f32x4{};
        mom[k] = in && l.momentum ? load4(l.momentum, from + r * l.cols + c0, LP_F32, vec4, left) : f32x4{};
    }
    if (l.dtype != LP_F32) {
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int r = r0 + k * dr;
            if (r < l.rows && left > 0) v[k] = load4(l.in, from + r * l.cols + c0, l.dtype, vec4, left);
        }
    }
    if (m != mp || n != np) {   // (rows and columns behind the matrix's)
        for (int i = threadIdx.x; i < mp * (np + 1); i += kThreads) g[i] = 0.0f;
        __syncthreads();
    }
    double norm = 0.0;
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
        const int r = r0 + k * dr;
        if (r >= l.rows || left <= 0) continue;
        if (l.momentum) {
            float* to = l.momentum + from + r * l.cols + c0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mom[k][e] = fmaf(a.mu, mom[k][e], v[k][e]);
                v[k][e] = a.nesterov ? fmaf(a.mu, mom[k][e], v[k][e]) : mom[k][e];
                if (!vec4 && e < left) to[e] = mom[k][e];
            }
            if (vec4) *(f32x4*)to = mom[k];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e >= left) continue;
            norm += (double)v[k][e] * (double)v[k][e];
            g[l.tall ? (c0 + e) * (np + 1) + r : r * (np + 1) + c0 + e] = v[k][e];
        }
    }
    for (int o = 32; o; o >>= 1) norm += __shfl_xor(norm, o);
    if (lane == 0) sums[wave] = norm;
    if (threadIdx.x < LP_ORTH_MAX_STEPS * 5) scales[threadIdx.x] = my_scale;
    __syncthreads();
    const Scale f = scale_of(sums[0] + sums[1] + sums[2] + sums[3], a.eps, a.load);
    if constexpr (LONG) {
        switch (mp / 32 * 16 + np / 32) {
            case 22: small_steps<1, 6>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 24: small_steps<1, 8>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 26: small_steps<1, 10>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 28: small_steps<1, 12>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 30: small_steps<1, 14>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 38: small_steps<2, 6>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 39: small_steps<2, 7>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
        }
    } else {
        switch (mp / 32 * 16 + np / 32) {
            case 17: small_steps<1, 1>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 18: small_steps<1, 2>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 19: small_steps<1, 3>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 20: small_steps<1, 4>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 34: small_steps<2, 2>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 35: small_steps<2, 3>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
            case 36: small_steps<2, 4>(a, l, a.steps, scales, X, XT, B, A, g, f, from); break;
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int pad(int v) { return (v + kPad - 1) / kPad * kPad; }

struct HostList {
    long long count;
    int rows, cols;
    const void* in;
    void* out;
    float* momentum;
    int dtype;
    bool small;   // one workgroup does all of a matrix
};

size_t matrix_halves(int rows, int cols)
{
    const size_t mp = pad(rows < cols ? rows : cols), np = pad(rows < cols ? cols : rows);
    return 8 * mp * np + 4 * mp * mp;
}

lp_status check_shape(long long count, int rows, int cols, int index)
{
    if (count < 0 || rows < 0 || cols < 0)
        return fail(LP_ERR_INVALID_ARG, "lists[" + std::to_string(index) + "]: count, rows and cols must be >= 0");
    if (rows > 65536 || cols > 65536 || count > (1 << 20))
        return fail(LP_ERR_UNSUPPORTED, "lists[" + std::to_string(index) + "]: at most 65536 rows or columns and 2^20 matrices");
    return LP_OK;
}

// Which matrices one workgroup does.  Those of at most 64 x 128 always; longer ones (41 us a call, however few) unless other lists of
// the call need the large matrices' launches anyway, where a few more tiles cost next to nothing: 500 matrices of 64 x 200 take 295
// us there and 93 in one workgroup each, so from about 100 on they are kept apart.
void choose_kernels(std::vector<HostList>* v)
{
    bool large = false;
    long long longer = 0;
    for (const HostList& q : *v) {
        if (!fits_one_workgroup(q.rows, q.cols)) large = true;
        else if (std::max(q.rows, q.cols) > kSmallN) longer += q.count;
    }
    for (HostList& q : *v)
        q.small = fits_one_workgroup(q.rows, q.cols) && (std::max(q.rows, q.cols) <= kSmallN || !large || longer >= 100);
}

// Workspace of a set of at most kMaxLists lists: the norms, then the matrices' planes.
size_t set_bytes(const std::vector<HostList>& v, size_t first, size_t end)
{
    size_t matrices = 0, planes = 0;
    for (size_t k = first; k < end; ++k) {
        if (v[k].small) continue;
        matrices += (size_t)v[k].count;
        planes += (size_t)v[k].count * align256(matrix_halves(v[k].rows, v[k].cols) * 2);
    }
    return matrices ? align256(matrices * kNormChunks * sizeof(double)) + align256(sizeof(Lists)) + planes : 0;
}


// How a set's A = X X^T is divided.
struct GramPlan {
    int tile, groups;
    int splits[kMaxLists], chunk;   // of the set's lists; 1: not divided
    long long parts;                // tiles of all parts; 0: no list is divided
};
GramPlan plan_gram(const std::vector<HostList>& v, size_t first, size_t end)
{
    GramPlan g;
    std::memset(&g, 0, sizeof(g));
    long long large = 0, steps = 0;
    for (size_t k = first; k < end; ++k) {
        if (v[k].small) continue;
        const long long mp = pad(v[k].rows < v[k].cols ? v[k].rows : v[k].cols), np = pad(v[k].rows < v[k].cols ? v[k].cols : v[k].rows);
        const long long t128 = (mp + 127) / 128, t64 = mp / 64;
        large += v[k].count * (t128 * (t128 + 1) / 2);
        steps += v[k].count * (t64 * (t64 + 1) / 2) * (np / kDepth);
    }
    for (int& s : g.splits) s = 1;
    if (large >= 2 * kUnits) {
        g.tile = 128;
        g.groups = 1;
        return g;
    }
    g.tile = 64;
    g.groups = 4;
    const long long even = (steps + 2 * kUnits - 1) / (2 * kUnits);
    g.chunk = (int)((even > 32 ? even + 3 : 32) / 4 * 4);   // (shortest parts of 16, 32, 64 steps: 279, 247, 265 us for the weights of ten convolutions)
    bool divided = false;
    for (size_t k = first; k < end; ++k) {
        if (v[k].small) continue;
        const long long mp = pad(v[k].rows < v[k].cols ? v[k].rows : v[k].cols), np = pad(v[k].rows < v[k].cols ? v[k].cols : v[k].rows);
        const int s = (int)((np / kDepth + g.chunk - 1) / g.chunk);
        g.splits[k - first] = s;
        g.parts += v[k].count * (mp / 64 * (mp / 64 + 1) / 2) * s;
        divided = divided || s > 1;
    }
    if (!divided) g.parts = 0;
    return g;
}

size_t all_bytes(const std::vector<HostList>& v)
{
    size_t most = 0;
    for (size_t k = 0; k < v.size(); k += kMaxLists) {
        const size_t end = v.size() < k + kMaxLists ? v.size() : k + kMaxLists;
        const GramPlan g = plan_gram(v, k, end);
        const size_t need = set_bytes(v, k, end) + (size_t)g.parts * g.tile * g.tile * sizeof(float);
        most = need > most ? need : most;
    }
    return most;
}

// max over lambda in [0, top] of |a + b lambda + c lambda^2|
double most_quadratic(double a, double b, double c, double top)
{
    double most = fmax(fabs(a), fabs(a + b * top + c * top * top));
    const double at = c != 0.0 ? -b / (2 * c) : -1.0;
    if (at > 0.0 && at < top) most = fmax(most, fabs(a + b * at + c * at * at));
    return most;
}
// max over s in [0, top] of |a s + b s^3 + c s^5|
double most_quintic(double a, double b, double c, double top)
{
    auto p = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
    double most = p(top);
    // the derivative a + 3 b l + 5 c l^2 at l = s^2
    double roots[2] = {-1.0, -1.0};
    if (c != 0.0) {
        const double disc = 9 * b * b - 20 * a * c;
        if (disc >= 0.0) {
            roots[0] = (-3 * b + sqrt(disc)) / (10 * c);
            roots[1] = (-3 * b - sqrt(disc)) / (10 * c);
        }
    } else if (b != 0.0) {
        roots[0] = -a / (3 * b);
    }
    for (double l : roots)
        if (l > 0.0 && l < top * top) most = fmax(most, p(sqrt(l)));
    return most;
}

double scale_for(double bound)   // the power of two that puts the bound (with 1 % for rounding) at or below 2^15
{
    int e;
    frexp(fmax(bound, 1e-30) * 1.01, &e);
    return ldexp(1.0, 15 - e);
}

lp_status make_plan(const lp_orth* o, Plan* plan)
{
    if (o->steps < 1 || o->steps > LP_ORTH_MAX_STEPS)
        return fail(LP_ERR_INVALID_ARG, "orth->steps must be in [1, LP_ORTH_MAX_STEPS]");
    if (!std::isfinite(o->eps) || o->eps < 0.0f) return fail(LP_ERR_INVALID_ARG, "orth->eps must be finite and >= 0");
    plan->steps = o->steps;
    double top = 1.0, ex = scale_for(top);
    plan->load = (float)ex;
    for (int k = 0; k < o->steps; ++k) {
        const double a = o->coeffs ? o->coeffs[3 * k] : 3.4445, b = o->coeffs ? o->coeffs[3 * k + 1] : -4.775,
                     c = o->coeffs ? o->coeffs[3 * k + 2] : 2.0315;
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c))
            return fail(LP_ERR_INVALID_ARG, "orth->coeffs must be finite");
        const double ea = scale_for(top * top), eb = scale_for(most_quadratic(a, b, c, top * top));
        plan->gram[k] = {(float)(ea / (ex * ex)), 0.0f, 0.0f, k & 1, 0};
        plan->poly[k] = {(float)(c * eb / (ea * ea)), (float)(a * eb), (float)(b * eb / ea), k & 1, 0};
        top = most_quintic(a, b, c, top);
        if (!(top <= 1024.0))
            return fail(LP_ERR_INVALID_ARG, "orth->coeffs let singular values leave [0, 1024] in step " + std::to_string(k));
        const double next = scale_for(top);
        const bool last = k + 1 == o->steps;
        plan->update[k] = {(float)((last ? 1.0 : next) / (eb * ex)), 0.0f, 0.0f, k & 1, (k + 1) & 1};
        ex = next;
    }
    return LP_OK;
}

lp_status launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LP_OK : fail(LP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// Numbers the workgroups of a launch: `tiles_of` gives those of one matrix.
constexpr int kMaxTiles = 1 << 23;   // workgroups of a launch (2^31 threads)
template <class F>
void number(Lists* a, LaunchOf which, F&& tiles_of)
{
    Launch& q = a->launch[which];
    int at = 0;
    for (int k = 0; k < kMaxLists; ++k) {
        q.all[k] = k < a->n ? at : INT_MAX;
        if (k < a->n) at += (q.tiles[k] = tiles_of(a->l[k])) * a->l[k].count;
    }
    q.total = at;
}

// The same for a product, lists of more `steps` first.
template <class F, class G>
void number_product(Lists* a, LaunchOf which, F&& tiles_of, G&& steps)
{
    number(a, which, tiles_of);
    Launch& q = a->launch[which];
    for (int k = 0; k < a->n; ++k) q.order[k] = k;
    std::sort(q.order, q.order + a->n, [&](int i, int j) { return steps(a->l[i]) != steps(a->l[j]) ? steps(a->l[i]) > steps(a->l[j]) : i < j; });
    for (int k = 0; k < kMaxLists; ++k) q.all[k] = k < a->n ? q.tiles[q.order[k]] * a->l[q.order[k]].count : 0;
}

// Workgroups of a product: eight times the most that an XCD has.
unsigned grid_of(const Lists& a, LaunchOf which)
{
    int most = 0;
    for (int x = 0; x < 8; ++x) {
        int sum = 0;
        for (int k = 0; k < a.n; ++k) {
            const int part = (x + 3 * k) & 7, all = a.launch[which].all[k];
            sum += (all * (part + 1) >> 3) - (all * part >> 3);
        }
        most = sum > most ? sum : most;
    }
    return 8u * (unsigned)most;
}

struct Muon {
    float lr_decay, mu, lr;
    int nesterov, scale;
};

lp_status run_set(const std::vector<HostList>& v, size_t first, size_t end, const Plan& plan, float eps, const Muon* muon,
                  void* workspace, hipStream_t s)
{
    Lists a;
    std::memset(&a, 0, sizeof(a));
    a.eps = eps;
    a.norms = (double*)workspace;
    if (muon) {
        a.lr_decay = muon->lr_decay;
        a.mu = muon->mu;
        a.nesterov = muon->nesterov;
    }
    size_t matrices = 0;
    for (size_t k = first; k < end; ++k)
        if (!v[k].small) matrices += (size_t)v[k].count;
    const size_t lists_at = align256(matrices * kNormChunks * sizeof(double));
    char* at = (char*)workspace + lists_at + align256(sizeof(Lists));
    const GramPlan gram = plan_gram(v, first, end);
    SmallCall smalls[2];   // up to 64 x 128, longer ones
    int lds[2] = {0, 0}, small_matrices[2] = {0, 0};
    for (SmallCall& small : smalls) {
        std::memset(&small, 0, sizeof(small));
        small.lr_decay = a.lr_decay; small.mu = a.mu; small.nesterov = a.nesterov; small.eps = eps;
        for (int k = 0; k < kMaxLists; ++k) small.first[k] = INT_MAX;
    }
    for (size_t k = first; k < end; ++k) {
        const HostList& q = v[k];
        const int tall = q.rows > q.cols, m = tall ? q.cols : q.rows, n = tall ? q.rows : q.cols;
        const bool aligned = (uintptr_t)q.in % 16 == 0 && (uintptr_t)q.momentum % 16 == 0;
        float step = 0.0f;
        if (muon) {
            const double ratio = (double)q.rows / q.cols;
            step = (float)(muon->lr * (muon->scale == LP_MUON_SCALE_ASPECT ? sqrt(ratio > 1.0 ? ratio : 1.0)
                                     : muon->scale == LP_MUON_SCALE_RMS ? 0.2 * sqrt((double)n) : 1.0));
        }
        if (q.small) {
            const int which = n > kSmallN;
            SmallCall& small = smalls[which];
            small.first[small.n] = small_matrices[which];
            small.l[small.n++] = {q.in, q.out, q.momentum, q.rows, q.cols, m, n, tall, q.dtype, aligned, step};
            small_matrices[which] += (int)q.count;
            lds[which] = std::max(lds[which], small_lds(pad32(m), small_columns(pad32(m), n)));
            continue;
        }
        List& l = a.l[a.n++];
        l.in = q.in; l.out = q.out; l.momentum = q.momentum; l.dtype = q.dtype; l.step = step;
        l.count = (int)q.count; l.rows = q.rows; l.cols = q.cols; l.tall = tall;
        l.m = m; l.n = n; l.mp = pad(m); l.np = pad(n);
        l.ws = (_Float16*)at;
        l.ws_stride = (long long)align256(matrix_halves(q.rows, q.cols) * 2) / 2;
        at += (size_t)l.ws_stride * 2 * q.count;
        l.vec4 = aligned && (long long)q.rows * q.cols % 4 == 0;
        l.splits = gram.splits[k - first];
        l.chunk = gram.chunk;
        l.first_matrix = a.matrices;
        a.matrices += l.count;
    }
    for (int which = 0; which < 2; ++which) {
        SmallCall& small = smalls[which];
        if (!small.n) continue;
        const void* kernel = which ? (const void*)orth_small_kernel<true> : (const void*)orth_small_kernel<false>;
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kSmallLds);   // (the same from every thread)
        if (e != hipSuccess) return fail(LP_ERR_HIP, std::string("hipFuncSetAttribute(orth_small_kernel): ") + hipGetErrorString(e));
        small.load = plan.load;
        small.steps = plan.steps;
        for (int k = 0; k < plan.steps; ++k) {
            const float w[5] = {plan.gram[k].acc, plan.poly[k].acc, plan.poly[k].diag, plan.poly[k].lin, plan.update[k].acc};
            std::memcpy(small.v[k], w, sizeof(w));
        }
        if (which) hipLaunchKernelGGL(orth_small_kernel<true>, dim3(small_matrices[which]), dim3(kThreads), lds[which], s, small);
        else hipLaunchKernelGGL(orth_small_kernel<false>, dim3(small_matrices[which]), dim3(kThreads), lds[which], s, small);
    }
    if (a.n == 0) return launched("orthogonalisation launch");
    a.parts = (float*)at;
    Lists* in_memory = (Lists*)((char*)workspace + lists_at);
    auto tiles = [](const List& l, int tile, bool half) {
        const int mt = (l.mp + tile - 1) / tile, nt = (l.np + tile - 1) / tile;
        return half ? mt * (mt + 1) / 2 : mt * nt;
    };
    number(&a, kOfNorm, [](const List& l) { return norm_chunks((long long)l.rows * l.cols); });   // (never more than the matrix has tiles)
    number(&a, kOfLoad, [](const List& l) { return (l.mp / 64) * (l.np / 64); });
    // How a product is divided.  Large tiles where they give every compute unit work.  Two small workgroups a unit overlap one's
    // ends with the other's products (B X of 340 tiles with sums of 64 .. 256: 19 us, in one large workgroup a unit 24, in 64 x 64
    // tiles 34); the long sums of A = X X^T are better halved inside a workgroup while there are fewer than two a unit (308 tiles:
    // 104 and 130 us).
    struct Shape { int tile, groups; };
    auto shape_of = [&](LaunchOf which, bool half) {
        const bool is_gram = which == kOfGram;
        auto steps = [&](const List& l) { return is_gram ? l.np : l.mp; };
        number_product(&a, which, [&](const List& l) { return tiles(l, 128, half); }, steps);
        if (a.launch[which].total >= (is_gram ? 2 : 1) * kUnits) return Shape{128, 1};
        if (is_gram && a.launch[which].total >= kUnits) return Shape{128, 2};
        number_product(&a, which, [&](const List& l) { return tiles(l, 64, half); }, steps);
        return Shape{64, 4};
    };
    // A = X X^T: where few tiles have long sums, these are divided among workgroups and joined by a second launch
    bool divided = false;
    for (int k = 0; k < a.n; ++k) divided = divided || a.l[k].splits > 1;
    Shape gram_shape = {64, 4};
    if (divided) {
        int first_part = 0;
        for (int k = 0; k < a.n; ++k) {
            a.l[k].first_part = first_part;
            first_part += a.l[k].count * tiles(a.l[k], 64, true) * a.l[k].splits;
        }
        auto steps = [](const List& l) { return std::min(l.chunk, l.np / kDepth); };
        number_product(&a, kOfGram, [&](const List& l) { return tiles(l, 64, true) * l.splits; }, steps);
        number_product(&a, kOfJoin, [&](const List& l) { return tiles(l, 64, true); }, steps);
    } else {
        gram_shape = shape_of(kOfGram, true);
    }
    const Shape poly_shape = shape_of(kOfPoly, true), update_shape = shape_of(kOfUpdate, false);
    const unsigned gram_grid = grid_of(a, kOfGram), join_grid = divided ? grid_of(a, kOfJoin) : 0, poly_grid = grid_of(a, kOfPoly),
                   update_grid = grid_of(a, kOfUpdate);
    hipLaunchKernelGGL(orth_norm_kernel, dim3(a.launch[kOfNorm].total), dim3(kThreads), 0, s, a, in_memory);
    hipLaunchKernelGGL(orth_load_kernel, dim3(a.launch[kOfLoad].total), dim3(kThreads), 0, s, in_memory, plan.load);
    auto product = [&](auto what, const Shape& shape, unsigned grid, const Step& step) {
        constexpr Product W = decltype(what)::value;
        if (shape.tile == 64) {
            hipLaunchKernelGGL((orth_product_kernel<W, 64, 4>), dim3(grid), dim3(512), 0, s, in_memory, step);
        } else if constexpr (W != kPart && W != kJoin) {
            if constexpr (W == kGram) {
                if (shape.groups == 2) {
                    hipLaunchKernelGGL((orth_product_kernel<W, 128, 2>), dim3(grid), dim3(512), 0, s, in_memory, step);
                    return;
                }
            }
            hipLaunchKernelGGL((orth_product_kernel<W, 128, 1>), dim3(grid), dim3(256), 0, s, in_memory, step);
        }
    };
    for (int k = 0; k < plan.steps; ++k) {
        if (divided) {
            product(std::integral_constant<Product, kPart>(), gram_shape, gram_grid, plan.gram[k]);
            product(std::integral_constant<Product, kJoin>(), gram_shape, join_grid, plan.gram[k]);
        } else {
            product(std::integral_constant<Product, kGram>(), gram_shape, gram_grid, plan.gram[k]);
        }
        product(std::integral_constant<Product, kPoly>(), poly_shape, poly_grid, plan.poly[k]);
        if (k + 1 < plan.steps) product(std::integral_constant<Product, kUpdate>(), update_shape, update_grid, plan.update[k]);
        else product(std::integral_constant<Product, kLast>(), update_shape, update_grid, plan.update[k]);
    }
    return launched("orthogonalisation launch");
}

// Whether something that is written lies over something else (but a result over its own list's input).
bool overlap(const std::vector<HostList>& v)
{
    struct Range {
        uintptr_t from, end;
        bool written;
    };
    std::vector<Range> ranges;
    ranges.reserve(3 * v.size());
    for (const HostList& q : v) {
        const uintptr_t bytes = (uintptr_t)q.count * q.rows * q.cols * (q.dtype == LP_F32 ? 4 : 2);
        auto add = [&](const void* p, bool written) { ranges.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written}); };
        add(q.out, true);
        if (q.momentum) add(q.momentum, true);
        if (q.momentum || q.in != q.out) add(q.in, false);
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t all_end = 0, written_end = 0;   // of the ranges before
    for (const Range& r : ranges) {
        if (r.from < (r.written ? all_end : written_end)) return true;
        all_end = std::max(all_end, r.end);
        if (r.written) written_end = std::max(written_end, r.end);
    }
    return false;
}

lp_status run(const std::vector<HostList>& v, const Plan& plan, float eps, const Muon* muon, void* workspace, size_t workspace_bytes,
              hipStream_t s)
{
    if (v.empty()) return LP_OK;
    const size_t need = all_bytes(v);
    if (need && (!workspace || workspace_bytes < need))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than the call's workspace_bytes function says");
    if (need && (uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    // (refused before anything is launched)
    if (overlap(v)) return fail(LP_ERR_INVALID_ARG, "what a list writes must not overlap another list's tensors or its own (but out may be in)");
    for (size_t k = 0; k < v.size(); k += kMaxLists) {
        double tiles = 0.0;
        for (size_t i = k; i < v.size() && i < k + kMaxLists; ++i)
            tiles += (double)v[i].count * (pad(v[i].rows) / 64) * (pad(v[i].cols) / 64);
        if (tiles > (double)kMaxTiles) return fail(LP_ERR_UNSUPPORTED, "too many matrices for one call");
    }
    for (size_t k = 0; k < v.size(); k += kMaxLists) {
        const lp_status st = run_set(v, k, v.size() < k + kMaxLists ? v.size() : k + kMaxLists, plan, eps, muon, workspace, s);
        if (st != LP_OK) return st;
    }
    return LP_OK;
}

lp_status collect(int32_t n, const lp_matrices* lists, bool pointers, std::vector<HostList>* v)
{
    if (n < 0) return fail(LP_ERR_INVALID_ARG, "n must be >= 0");
    if (n > 0 && !lists) return fail(LP_ERR_INVALID_ARG, "lists must not be NULL");
    for (int k = 0; k < n; ++k) {
        const lp_matrices& q = lists[k];
        const lp_status st = check_shape(q.count, q.rows, q.cols, k);
        if (st != LP_OK) return st;
        if (q.dtype != LP_F32 && q.dtype != LP_BF16 && q.dtype != LP_F16)
            return fail(LP_ERR_INVALID_ARG, "lists[" + std::to_string(k) + "].dtype must be LP_F32, LP_BF16 or LP_F16");
        if (!q.count || !q.rows || !q.cols) continue;
        if (pointers && (!q.in || !q.out)) return fail(LP_ERR_INVALID_ARG, "lists[" + std::to_string(k) + "] has a NULL tensor");
        v->push_back({q.count, q.rows, q.cols, q.in, q.out, nullptr, q.dtype, false});
    }
    choose_kernels(v);
    return LP_OK;
}

lp_status collect(int32_t n, const lp_muon_weights* lists, bool pointers, std::vector<HostList>* v)
{
    if (n < 0) return fail(LP_ERR_INVALID_ARG, "n must be >= 0");
    if (n > 0 && !lists) return fail(LP_ERR_INVALID_ARG, "lists must not be NULL");
    for (int k = 0; k < n; ++k) {
        const lp_muon_weights& q = lists[k];
        const lp_status st = check_shape(q.count, q.rows, q.cols, k);
        if (st != LP_OK) return st;
        if (!q.count || !q.rows || !q.cols) continue;
        if (pointers && (!q.weight || !q.grad || !q.momentum))
            return fail(LP_ERR_INVALID_ARG, "lists[" + std::to_string(k) + "] has a NULL tensor");
        v->push_back({q.count, q.rows, q.cols, q.grad, q.weight, q.momentum, LP_F32, false});
    }
    choose_kernels(v);
    return LP_OK;
}

}  // namespace

}  // namespace lp

extern "C" {

lp_status lp_orthogonalize_workspace_bytes(int32_t n, const lp_matrices* lists, size_t* bytes)
try {
    std::vector<lp::HostList> v;
    const lp_status st = lp::collect(n, lists, false, &v);
    if (st != LP_OK) return st;
    if (!bytes) return lp::fail(LP_ERR_INVALID_ARG, "bytes must not be NULL");
    *bytes = lp::all_bytes(v);
    return LP_OK;
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_muon_workspace_bytes(int32_t n, const lp_muon_weights* lists, size_t* bytes)
try {
    std::vector<lp::HostList> v;
    const lp_status st = lp::collect(n, lists, false, &v);
    if (st != LP_OK) return st;
    if (!bytes) return lp::fail(LP_ERR_INVALID_ARG, "bytes must not be NULL");
    *bytes = lp::all_bytes(v);
    return LP_OK;
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_orthogonalize(int32_t n, const lp_matrices* lists, const lp_orth* orth, void* workspace, size_t workspace_bytes,
                           void* stream)
try {
    if (!orth) return lp::fail(LP_ERR_INVALID_ARG, "orth must not be NULL");
    std::vector<lp::HostList> v;
    lp_status st = lp::collect(n, lists, true, &v);
    if (st != LP_OK) return st;
    lp::Plan plan;
    if ((st = lp::make_plan(orth, &plan)) != LP_OK) return st;
    return lp::run(v, plan, orth->eps, nullptr, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_muon_step(int32_t n, const lp_muon_weights* lists, const lp_muon* muon, void* workspace, size_t workspace_bytes, void* stream)
try {
    if (!muon) return lp::fail(LP_ERR_INVALID_ARG, "muon must not be NULL");
    std::vector<lp::HostList> v;
    lp_status st = lp::collect(n, lists, true, &v);
    if (st != LP_OK) return st;
    if (!std::isfinite(muon->lr) || !std::isfinite(muon->momentum) || !std::isfinite(muon->weight_decay))
        return lp::fail(LP_ERR_INVALID_ARG, "muon->lr, momentum and weight_decay must be finite");
    if (muon->nesterov != 0 && muon->nesterov != 1) return lp::fail(LP_ERR_INVALID_ARG, "muon->nesterov must be 0 or 1");
    if (muon->scale < LP_MUON_SCALE_NONE || muon->scale > LP_MUON_SCALE_RMS)
        return lp::fail(LP_ERR_INVALID_ARG, "muon->scale must be an lp_muon_scale");
    lp::Plan plan;
    if ((st = lp::make_plan(&muon->orth, &plan)) != LP_OK) return st;
    const lp::Muon m = {(float)(1.0 - (double)muon->lr * (double)muon->weight_decay), muon->momentum, muon->lr, muon->nesterov, muon->scale};
    return lp::run(v, plan, muon->orth.eps, &m, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

}  // extern "C"
