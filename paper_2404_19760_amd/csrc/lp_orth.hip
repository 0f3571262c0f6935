// Orthogonalised updates of weight matrices (Newton-Schulz products) and the optimiser step built on them.
//
//     X_0 = G / (||G||_F + eps),   A = X X^T,   B = a I + b A + c A A,   X <- B X     (X: m x n, m <= n)
//
// Precision: the products magnify what lies in the directions of small singular values (3.44 times a step), so operands of 8
// or 11 bits would leave 1e-3 in the result.  An operand is kept as two fp16 numbers, hi and lo = the rest, at a power-of-two
// scale: 22 bits.  Three matrix products (hi hi + hi lo + lo hi) with fp32 accumulation then have the error of fp32 products
// (measured against 64 bits: as fp32 torch products, 1e-6 .. 7e-6 over five steps) at 16/3 of the fp32 matrix rate.
// fp16 reaches to 65504: the host follows how far singular values can have got in every step (`Plan`) and scales each operand so
// that its bound lies below 2^15; an entry of a matrix is never larger than its largest singular value.
//
// What bounds it: matrix instructions for matrices from some hundreds of rows on, launches below.  X is kept in both orders (X
// and X^T), so that both operands of every product run along memory: A = X X^T from rows of X, A A from rows of A (A is
// symmetric), B X from rows of B and rows of X^T.  A and B are symmetric: only tiles on and above the diagonal are computed,
// and written twice.  a I is added into B, so that B X is all of the step.  Matrices of all lists go through one launch per
// product.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <vector>

#include "lp_kernels.h"

namespace lp {

namespace {

using half8 = _Float16 __attribute__((ext_vector_type(8)));
using half4 = _Float16 __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kMaxLists = 16;     // lists of one set of launches (their descriptors travel as kernel arguments)
constexpr int kPad = 64;          // rows and columns of operands are padded to this
constexpr int kNormChunks = 64;   // partial sums of a matrix's norm

// One list of matrices on the device side.  Layout of a matrix's workspace, in halves from `ws` + i `ws_stride`:
// four X planes of mp np (X hi, X lo, X^T hi, X^T lo) twice, then four planes of mp mp (A hi, lo, B hi, lo).
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
    int first_tile;     // of the launch
    int tiles;          // of one matrix
};

struct Lists {
    int n, matrices, total_tiles;
    float lr_decay;     // 1 - lr weight_decay
    float mu;
    int nesterov;
    float eps;
    double* norms;      // [matrices][kNormChunks]
    List l[kMaxLists];
};

__device__ __forceinline__ float load_value(const void* p, size_t i, int dtype)
{
    if (dtype == LP_F32) return ((const float*)p)[i];
    if (dtype == LP_BF16) return (float)((const __bf16*)p)[i];
    return (float)((const _Float16*)p)[i];
}
__device__ __forceinline__ void store_value(void* p, size_t i, int dtype, float v)
{
    if (dtype == LP_F32) ((float*)p)[i] = v;
    else if (dtype == LP_BF16) ((__bf16*)p)[i] = (__bf16)v;
    else ((_Float16*)p)[i] = (_Float16)v;
}

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// The list and the matrix of it that `tile` belongs to, and the tile within the matrix.
__device__ __forceinline__ const List& find(const Lists& a, int tile, int& matrix, int& local)
{
    int k = 0;
    while (k + 1 < a.n && tile >= a.l[k + 1].first_tile) ++k;
    const int rest = tile - a.l[k].first_tile;
    matrix = rest / a.l[k].tiles;
    local = rest - matrix * a.l[k].tiles;
    return a.l[k];
}

// Sums of squares in 64 bits (so that no gradient is too large or too small), one workgroup a (matrix, chunk); the optimiser
// step updates the momentum on the way.
__global__ __launch_bounds__(kThreads) void orth_norm_kernel(Lists a)
{
    __shared__ double lds[4];
    int matrix, chunk;
    const List& l = find(a, blockIdx.x, matrix, chunk);
    const long long size = (long long)l.rows * l.cols, from = (long long)matrix * size;
    double sum = 0.0;
    for (long long i = (long long)chunk * kThreads + threadIdx.x; i < size; i += (long long)l.tiles * kThreads) {
        float v = load_value(l.in, from + i, l.dtype);
        if (l.momentum) {
            const float mom = fmaf(a.mu, l.momentum[from + i], v);
            l.momentum[from + i] = mom;
            v = a.nesterov ? fmaf(a.mu, mom, v) : mom;
        }
        sum += (double)v * (double)v;
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.norms[(size_t)(l.first_matrix + matrix) * kNormChunks + chunk] = lds[0] + lds[1] + lds[2] + lds[3];
}

// X_0 and its transpose as hi and lo parts, padded with zeros: one workgroup a 64 x 64 tile of rows x cols.
__global__ __launch_bounds__(kThreads) void orth_load_kernel(Lists a, int chunks_shift, float scale)
{
    __shared__ _Float16 th[64 * 66], tl[64 * 66];
    __shared__ double factor;   // (in 64 bits: no gradient is too large or too small)
    int matrix, local;
    const List& l = find(a, blockIdx.x, matrix, local);
    if (threadIdx.x < 64) {
        double v = 0.0;
        const long long size = (long long)l.rows * l.cols;
        const int chunks = (int)min((long long)kNormChunks, (size + (1 << chunks_shift) - 1) >> chunks_shift);
        if ((int)threadIdx.x < chunks) v = a.norms[(size_t)(l.first_matrix + matrix) * kNormChunks + threadIdx.x];
        for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
        const double norm = sqrt(v);
        if (threadIdx.x == 0) factor = norm == 0.0 ? 0.0 : (double)scale / (norm + (double)a.eps);
    }
    __syncthreads();
    const double f = factor;
    const int rp = l.tall ? l.np : l.mp, cp = l.tall ? l.mp : l.np;   // padded rows and columns of G
    const int tr = local / (cp / 64), tc = local - tr * (cp / 64);
    const long long from = (long long)matrix * l.rows * l.cols;
    _Float16* ws = l.ws + (size_t)matrix * l.ws_stride;
    const size_t plane = (size_t)l.mp * l.np;
    _Float16* same = ws + (l.tall ? 2 * plane : 0);    // the planes in the order of G
    _Float16* other = ws + (l.tall ? 0 : 2 * plane);   // the planes of its transpose
    const int c = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        const int gr = tr * 64 + r, gc = tc * 64 + c;
        float v = 0.0f;
        if (gr < l.rows && gc < l.cols) {
            const size_t i = from + (size_t)gr * l.cols + gc;
            v = load_value(l.in, i, l.dtype);
            if (l.momentum) v = a.nesterov ? fmaf(a.mu, l.momentum[i], v) : l.momentum[i];
        }
        _Float16 hi, lo;
        split((float)((double)v * f), hi, lo);
        same[(size_t)gr * cp + gc] = hi;
        same[plane + (size_t)gr * cp + gc] = lo;
        th[r * 66 + c] = hi;
        tl[r * 66 + c] = lo;
    }
    __syncthreads();
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        const size_t at = (size_t)(tc * 64 + r) * rp + tr * 64 + c;
        other[at] = th[c * 66 + r];
        other[plane + at] = tl[c * 66 + r];
    }
}

enum Product { kGram, kPoly, kUpdate, kLast };

// Scales of one step: what the accumulator is multiplied with, and the polynomial's coefficients at B's scale.
struct Step {
    float acc;          // kGram, kUpdate: scale of the result over the operands'; kLast: 1 over the operands'; kPoly: c's factor
    float diag, lin;    // kPoly: a and b at B's scale
    int from, to;       // which of the two X's is read, written
};

constexpr int kTile = 64, kDepth = 32;

// One workgroup of four waves a 64 x 64 tile of P Q^T, a wave 32 x 32 of it.
template <Product WHAT>
__global__ __launch_bounds__(kThreads) void orth_product_kernel(Lists a, Step s)
{
    __shared__ alignas(16) _Float16 lds[4][kTile * (kDepth + 8)];   // P hi, P lo, Q hi, Q lo; rows padded against bank conflicts
    constexpr int kRow = kDepth + 8;
    int matrix, local;
    const List& l = find(a, blockIdx.x, matrix, local);
    _Float16* ws = l.ws + (size_t)matrix * l.ws_stride;
    const size_t plane = (size_t)l.mp * l.np, square = (size_t)l.mp * l.mp;
    _Float16* x = ws + s.from * 4 * plane;
    _Float16* A = ws + 8 * plane;
    _Float16* B = A + 2 * square;
    int ti, tj;
    const int mt = l.mp / kTile, nt = l.np / kTile;
    if (WHAT == kGram || WHAT == kPoly) {   // tiles on and above the diagonal, row by row
        ti = 0;
        int rest = local;
        while (rest >= mt - ti) rest -= mt - ti++;
        tj = ti + rest;
    } else {
        ti = local / nt;
        tj = local - ti * nt;
    }
    const _Float16 *p, *q;
    size_t p_lo, q_lo;
    int K;
    if (WHAT == kGram) { p = q = x; p_lo = q_lo = plane; K = l.np; }
    else if (WHAT == kPoly) { p = q = A; p_lo = q_lo = square; K = l.mp; }
    else { p = B; q = x + 2 * plane; p_lo = square; q_lo = plane; K = l.mp; }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wi = wave >> 1, wj = wave & 1, l32 = lane & 31, h = lane >> 5;
    f32x16 acc = {};
    const int sr = threadIdx.x >> 2, sc = (threadIdx.x & 3) * 8;   // a thread stages 8 halves of a row of each plane
    const size_t pat = (size_t)(ti * kTile + sr) * K + sc, qat = (size_t)(tj * kTile + sr) * K + sc;
    for (int k = 0; k < K; k += kDepth) {
        const half8 v0 = *(const half8*)(p + pat + k), v1 = *(const half8*)(p + p_lo + pat + k);
        const half8 v2 = *(const half8*)(q + qat + k), v3 = *(const half8*)(q + q_lo + qat + k);
        __syncthreads();
        *(half8*)&lds[0][sr * kRow + sc] = v0;
        *(half8*)&lds[1][sr * kRow + sc] = v1;
        *(half8*)&lds[2][sr * kRow + sc] = v2;
        *(half8*)&lds[3][sr * kRow + sc] = v3;
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kDepth; kk += 16) {
            const int pa = (wi * 32 + l32) * kRow + kk + 8 * h, qa = (wj * 32 + l32) * kRow + kk + 8 * h;
            const half8 ph = *(const half8*)&lds[0][pa], pl = *(const half8*)&lds[1][pa];
            const half8 qh = *(const half8*)&lds[2][qa], ql = *(const half8*)&lds[3][qa];
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
        }
    }
    // value e of a lane: row 8 (e / 4) + 4 h + e % 4, column l32 of the wave's 32 x 32
    const int i0 = ti * kTile + wi * 32, j = tj * kTile + wj * 32 + l32;
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
        half4 hi, lo;
        const int ib = i0 + 8 * e4 + 4 * h;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = ib + e;
            float v = acc[4 * e4 + e] * s.acc;
            if (WHAT == kPoly) {
                const size_t at = (size_t)i * l.mp + j;
                v = fmaf(s.lin, (float)A[at] + (float)A[square + at], v);
                if (i == j && i < l.m) v += s.diag;
            }
            if (WHAT == kLast) {
                if (i < l.m && j < l.n) {
                    const size_t at = (size_t)matrix * l.rows * l.cols + (l.tall ? (size_t)j * l.cols + i : (size_t)i * l.cols + j);
                    if (l.momentum) {
                        float* w = (float*)l.out + at;
                        *w = fmaf(-l.step, v, a.lr_decay * *w);
                    } else {
                        store_value(l.out, at, l.dtype, v);
                    }
                }
                continue;
            }
            _Float16 vh, vl;
            split(v, vh, vl);
            hi[e] = vh;
            lo[e] = vl;
        }
        if (WHAT == kLast) continue;
        // rows as they come (32 lanes, 64 bytes), and 4 neighbours of the transpose in one store
        _Float16* direct = WHAT == kGram ? A : WHAT == kPoly ? B : ws + s.to * 4 * plane;
        const size_t lo_at = WHAT == kUpdate ? plane : square;
        _Float16* trans = WHAT == kUpdate ? direct + 2 * plane : direct;
        const int width = WHAT == kUpdate ? l.np : l.mp;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (WHAT != kUpdate && ti == tj) break;   // (a tile on the diagonal is its own transpose)
            direct[(size_t)(ib + e) * width + j] = hi[e];
            direct[lo_at + (size_t)(ib + e) * width + j] = lo[e];
        }
        *(half4*)&trans[(size_t)j * l.mp + ib] = hi;
        *(half4*)&trans[lo_at + (size_t)j * l.mp + ib] = lo;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int pad(int v) { return (v + kPad - 1) / kPad * kPad; }
constexpr int kChunkShift = 14;   // values of a partial sum of the norm

struct HostList {
    long long count;
    int rows, cols;
    const void* in;
    void* out;
    float* momentum;
    int dtype;
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

// Workspace of a set of at most kMaxLists lists: the norms, then the matrices' planes.
size_t set_bytes(const std::vector<HostList>& v, size_t first, size_t end)
{
    size_t matrices = 0, planes = 0;
    for (size_t k = first; k < end; ++k) {
        matrices += (size_t)v[k].count;
        planes += (size_t)v[k].count * align256(matrix_halves(v[k].rows, v[k].cols) * 2);
    }
    return align256(matrices * kNormChunks * sizeof(double)) + planes;
}

size_t all_bytes(const std::vector<HostList>& v)
{
    size_t most = 0;
    for (size_t k = 0; k < v.size(); k += kMaxLists) {
        const size_t need = set_bytes(v, k, v.size() < k + kMaxLists ? v.size() : k + kMaxLists);
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

// Scales of all steps from the bounds of what the operands can hold.
struct Plan {
    float load;   // of X_0
    Step gram[LP_ORTH_MAX_STEPS], poly[LP_ORTH_MAX_STEPS], update[LP_ORTH_MAX_STEPS];
    int steps;
};

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
void number(Lists* a, F&& tiles_of)
{
    int at = 0;
    for (int k = 0; k < a->n; ++k) {
        a->l[k].first_tile = at;
        a->l[k].tiles = tiles_of(a->l[k]);
        at += a->l[k].tiles * a->l[k].count;
    }
    a->total_tiles = at;
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
    for (size_t k = first; k < end; ++k) matrices += (size_t)v[k].count;
    char* at = (char*)workspace + align256(matrices * kNormChunks * sizeof(double));
    for (size_t k = first; k < end; ++k) {
        List& l = a.l[a.n++];
        const HostList& q = v[k];
        l.in = q.in; l.out = q.out; l.momentum = q.momentum; l.dtype = q.dtype;
        l.count = (int)q.count; l.rows = q.rows; l.cols = q.cols;
        l.tall = q.rows > q.cols;
        l.m = l.tall ? q.cols : q.rows; l.n = l.tall ? q.rows : q.cols;
        l.mp = pad(l.m); l.np = pad(l.n);
        l.ws = (_Float16*)at;
        l.ws_stride = (long long)align256(matrix_halves(q.rows, q.cols) * 2) / 2;
        at += (size_t)l.ws_stride * 2 * q.count;
        l.first_matrix = a.matrices;
        a.matrices += l.count;
        if (muon) {
            const double ratio = (double)q.rows / q.cols, larger = q.rows > q.cols ? q.rows : q.cols;
            const double scale = muon->scale == LP_MUON_SCALE_ASPECT ? sqrt(ratio > 1.0 ? ratio : 1.0)
                               : muon->scale == LP_MUON_SCALE_RMS ? 0.2 * sqrt(larger) : 1.0;
            l.step = (float)(muon->lr * scale);
        }
    }
    auto norm_chunks = [](const List& l) {
        const long long c = ((long long)l.rows * l.cols + (1 << kChunkShift) - 1) >> kChunkShift;
        return (int)(c < kNormChunks ? c : kNormChunks);   // (never more than the matrix has tiles)
    };
    auto all_tiles = [](const List& l) { return (l.mp / kTile) * (l.np / kTile); };
    auto half_tiles = [](const List& l) { const int t = l.mp / kTile; return t * (t + 1) / 2; };
    number(&a, norm_chunks);
    hipLaunchKernelGGL(orth_norm_kernel, dim3(a.total_tiles), dim3(kThreads), 0, s, a);
    number(&a, all_tiles);
    hipLaunchKernelGGL(orth_load_kernel, dim3(a.total_tiles), dim3(kThreads), 0, s, a, kChunkShift, plan.load);
    for (int k = 0; k < plan.steps; ++k) {
        number(&a, half_tiles);
        hipLaunchKernelGGL((orth_product_kernel<kGram>), dim3(a.total_tiles), dim3(kThreads), 0, s, a, plan.gram[k]);
        hipLaunchKernelGGL((orth_product_kernel<kPoly>), dim3(a.total_tiles), dim3(kThreads), 0, s, a, plan.poly[k]);
        number(&a, all_tiles);
        if (k + 1 < plan.steps)
            hipLaunchKernelGGL((orth_product_kernel<kUpdate>), dim3(a.total_tiles), dim3(kThreads), 0, s, a, plan.update[k]);
        else
            hipLaunchKernelGGL((orth_product_kernel<kLast>), dim3(a.total_tiles), dim3(kThreads), 0, s, a, plan.update[k]);
    }
    return launched("orthogonalisation launch");
}

lp_status run(const std::vector<HostList>& v, const Plan& plan, float eps, const Muon* muon, void* workspace, size_t workspace_bytes,
              hipStream_t s)
{
    if (v.empty()) return LP_OK;
    if (!workspace || workspace_bytes < all_bytes(v))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than the call's workspace_bytes function says");
    if ((uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    // (refused before anything is launched)
    for (size_t k = 0; k < v.size(); k += kMaxLists) {
        double tiles = 0.0;
        for (size_t i = k; i < v.size() && i < k + kMaxLists; ++i)
            tiles += (double)v[i].count * (pad(v[i].rows) / kTile) * (pad(v[i].cols) / kTile);
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
        v->push_back({q.count, q.rows, q.cols, q.in, q.out, nullptr, q.dtype});
    }
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
        v->push_back({q.count, q.rows, q.cols, q.grad, q.weight, q.momentum, LP_F32});
    }
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
