// The norm of all gradients of a step together, and the gradients brought under a largest norm.
//
//     norm = sqrt(sum of g^2),   out = g min(1, max_norm / (norm + eps))
//
// What bounds it: memory, and launches for a small decoder's gradients.  A sum over everything stands between reading a value and
// using it.  Up to 32 Ki values stay in the registers of one workgroup meanwhile (one launch).  More are passed over twice: workgroups
// leave their sums in the workspace, and those of the second pass add all of them up before they scale their part; they go through the
// values from the end backwards, so that what the first pass read last is still in the Infinity Cache.  Where the values are more than
// it holds, results go past it, so as not to drive out what is yet to be read (150 million values in fp32, 0.6 GB: 312 us; with
// ordinary stores 344, from the start on 352).
//
// Squares and sums are fp64: the square of an fp32 value is exact there and neither overflows nor vanishes, and memory is far slower than
// the two instructions a value.  The order of the sums depends on the sizes alone.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <vector>

#include "lp_kernels.h"

namespace lp {

namespace {

constexpr int kThreads = 256;
constexpr int kSmallThreads = 1024;
constexpr int kSmallTensors = 8, kSmallSlots = 8;                  // one workgroup: tensors, slots of four values a thread
constexpr int kSetTensors = 64;                                    // tensors of one launch (their list is a kernel argument)
constexpr long long kLeast = 4096;                                 // values of a part, at least
constexpr int kJoinAtOnce = 4096;                                  // sums that every workgroup of the second pass adds up itself

struct TensorDev {
    const void* in;
    void* out;
    long long size;
    int first;   // its first part, or slot, among the set's
    int dtype;
};

template <int MAX>
struct Set {
    TensorDev t[MAX];
    int n, items;       // tensors; parts, or slots
    int before;         // parts of the sets before this one
    long long chunk;    // values of a part
};

// What is done with the sum of all squares.
struct Clip {
    float* norm;
    float max_norm, eps;
    int scale;   // 0: the norm alone
};

__device__ __forceinline__ double factor_of(double squares, const Clip& c)
{
    const double norm = sqrt(squares), f = (double)c.max_norm / (norm + (double)c.eps);
    return f >= 1.0 || norm == 0.0 ? 1.0 : f;   // (NaN stays NaN)
}
// Whether a factor has fewer bits in fp32, or none: norms beyond 1e38 times the largest one.  It is applied in fp64 then.
__device__ __forceinline__ bool is_tiny(double factor) { return factor > 0.0 && factor < (double)FLT_MIN; }

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
template <class T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

__device__ __forceinline__ void add_square(double& sum, float v) { sum = fma((double)v, (double)v, sum); }

// The sum over the workgroup, for all of its threads.
template <int THREADS>
__device__ __forceinline__ double all_of(double v, double* lds)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) sum += lds[w];
    return sum;
}

template <int MAX>
__device__ __forceinline__ int tensor_of(const Set<MAX>& a, int item)
{
    int lo = 0, hi = a.n - 1;   // the last one that starts at or before the item
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.t[mid].first <= item) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Values in front of the first 16-byte boundary.
template <class T>
__device__ __forceinline__ long long head_of(const T* p, long long count)
{
    const long long head = ((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T);
    return head < count ? head : count;
}

template <class T>
__device__ __forceinline__ double squares_of(const T* p, long long count)
{
    constexpr int V = 16 / sizeof(T), U = 4;
    using P = Pack<T, V>;
    double sum[2] = {0.0, 0.0};
    const long long head = head_of(p, count), packs = (count - head) / V, tail = head + packs * V;
    const P* body = (const P*)(p + head);
    long long i = threadIdx.x;
    for (; i + (U - 1) * kThreads < packs; i += U * kThreads) {
        P v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = body[i + u * kThreads];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < V; ++j) add_square(sum[j & 1], (float)v[u].v[j]);
    }
    for (; i < packs; i += kThreads) {
        const P v = body[i];
#pragma unroll
        for (int j = 0; j < V; ++j) add_square(sum[j & 1], (float)v.v[j]);
    }
    if (threadIdx.x < head) add_square(sum[0], (float)p[threadIdx.x]);
    if (threadIdx.x < count - tail) add_square(sum[1], (float)p[tail + threadIdx.x]);
    return sum[0] + sum[1];
}

template <bool PAST_CACHE, class T>
__device__ __forceinline__ void scale_part(const T* in, T* out, long long count, float factor)
{
    constexpr int V = 16 / sizeof(T), U = 4;
    using P = Pack<T, V>;
    if (((uintptr_t)in & 15) != ((uintptr_t)out & 15)) {   // no 16-byte boundaries in common
        for (long long i = threadIdx.x; i < count; i += kThreads) out[i] = (T)((float)in[i] * factor);
        return;
    }
    const long long head = head_of(in, count), packs = (count - head) / V, tail = head + packs * V;
    const P* body = (const P*)(in + head);
    P* to = (P*)(out + head);
    auto scaled = [&](P v) {
#pragma unroll
        for (int j = 0; j < V; ++j) v.v[j] = (T)((float)v.v[j] * factor);   // rounded once
        return v;
    };
    long long i = threadIdx.x;
    for (; i + (U - 1) * kThreads < packs; i += U * kThreads) {
        P v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = body[i + u * kThreads];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const P r = scaled(v[u]);
            if (PAST_CACHE) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), (u32x4*)&to[i + u * kThreads]);
            else to[i + u * kThreads] = r;
        }
    }
    for (; i < packs; i += kThreads) to[i] = scaled(body[i]);
    if (threadIdx.x < head) out[threadIdx.x] = (T)((float)in[threadIdx.x] * factor);
    if (threadIdx.x < count - tail) out[tail + threadIdx.x] = (T)((float)in[tail + threadIdx.x] * factor);
}

template <class T>
__device__ __forceinline__ void scale_exactly(const T* in, T* out, long long count, double factor)
{
    for (long long i = threadIdx.x; i < count; i += kThreads) out[i] = (T)(float)((double)in[i] * factor);
}

// One workgroup a part: its sum of squares.
template <int MAX>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(Set<MAX> a, double* parts)
{
    __shared__ double lds[kThreads / 64];
    const int k = tensor_of(a, blockIdx.x);
    const TensorDev& t = a.t[k];
    const long long at = (blockIdx.x - t.first) * a.chunk, count = min(a.chunk, t.size - at);
    double sum;
    if (t.dtype == LP_F32) sum = squares_of((const float*)t.in + at, count);
    else if (t.dtype == LP_BF16) sum = squares_of((const __bf16*)t.in + at, count);
    else sum = squares_of((const _Float16*)t.in + at, count);
    sum = all_of<kThreads>(sum, lds);
    if (threadIdx.x == 0) parts[a.before + blockIdx.x] = sum;
}

// The sum of the parts, for all threads of the workgroup; it needs no other workgroup's result than the parts.
template <int THREADS>
__device__ __forceinline__ double all_parts(const double* parts, int n, double* lds)
{
    double sum = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < n; i += THREADS) sum += parts[i];
    return all_of<THREADS>(sum, lds);
}

// One workgroup: the parts' sum into the place of `total` (NULL: none), and the norm.
__global__ __launch_bounds__(kSmallThreads) void grad_join_kernel(const double* parts, int n, double* total, float* norm)
{
    __shared__ double lds[kSmallThreads / 64];
    const double sum = all_parts<kSmallThreads>(parts, n, lds);
    if (threadIdx.x) return;
    if (total) *total = sum;
    *norm = (float)sqrt(sum);
}

// PAST_CACHE: results are stored past the caches.
template <bool PAST_CACHE, int MAX>
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Set<MAX> a, const double* parts, int n, Clip c, int write_norm)
{
    __shared__ double lds[kThreads / 64];
    const double sum = all_parts<kThreads>(parts, n, lds);
    if (write_norm && blockIdx.x == 0 && threadIdx.x == 0) *c.norm = (float)sqrt(sum);
    const double exact = factor_of(sum, c);
    const float factor = (float)exact;
    const int item = a.items - 1 - blockIdx.x, k = tensor_of(a, item);
    const TensorDev& t = a.t[k];
    if (factor == 1.0f && t.in == t.out) return;   // (nothing changes)
    const long long at = (item - t.first) * a.chunk, count = min(a.chunk, t.size - at);
    if (is_tiny(exact)) {
        if (t.dtype == LP_F32) scale_exactly((const float*)t.in + at, (float*)t.out + at, count, exact);
        else if (t.dtype == LP_BF16) scale_exactly((const __bf16*)t.in + at, (__bf16*)t.out + at, count, exact);
        else scale_exactly((const _Float16*)t.in + at, (_Float16*)t.out + at, count, exact);
        return;
    }
    if (t.dtype == LP_F32) scale_part<PAST_CACHE>((const float*)t.in + at, (float*)t.out + at, count, factor);
    else if (t.dtype == LP_BF16) scale_part<PAST_CACHE>((const __bf16*)t.in + at, (__bf16*)t.out + at, count, factor);
    else scale_part<PAST_CACHE>((const _Float16*)t.in + at, (_Float16*)t.out + at, count, factor);
}

// Everything in one workgroup: slots of four neighbouring values, held between the sum and the scaling.
template <class T>
__device__ __forceinline__ void load_slot(const TensorDev& t, long long at, float (&v)[4])
{
    const T* p = (const T*)t.in + at;
    if (at + 4 <= t.size && ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0) {
        const Pack<T, 4> q = *(const Pack<T, 4>*)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)q.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = at + j < t.size ? (float)p[j] : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void store_slot(const TensorDev& t, long long at, const float (&v)[4], float factor)
{
    T* p = (T*)t.out + at;
    if (at + 4 <= t.size && ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0) {
        Pack<T, 4> q;
#pragma unroll
        for (int j = 0; j < 4; ++j) q.v[j] = (T)(v[j] * factor);
        *(Pack<T, 4>*)p = q;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (at + j < t.size) p[j] = (T)(v[j] * factor);
    }
}

__global__ __launch_bounds__(kSmallThreads) void grad_small_kernel(Set<kSmallTensors> a, Clip c)
{
    __shared__ double lds[kSmallThreads / 64];
    float v[kSmallSlots][4];
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < kSmallSlots; ++s) {
        const int slot = s * kSmallThreads + threadIdx.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[s][j] = 0.0f;
        if (slot >= a.items) continue;
        const TensorDev& t = a.t[tensor_of(a, slot)];
        const long long at = 4ll * (slot - t.first);
        if (t.dtype == LP_F32) load_slot<float>(t, at, v[s]);
        else if (t.dtype == LP_BF16) load_slot<__bf16>(t, at, v[s]);
        else load_slot<_Float16>(t, at, v[s]);
    }
#pragma unroll
    for (int s = 0; s < kSmallSlots; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) add_square(sum, v[s][j]);
    sum = all_of<kSmallThreads>(sum, lds);
    if (threadIdx.x == 0) *c.norm = (float)sqrt(sum);
    if (!c.scale) return;
    const double exact = factor_of(sum, c);
    float factor = (float)exact;
    if (is_tiny(exact)) {
#pragma unroll
        for (int s = 0; s < kSmallSlots; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[s][j] = (float)((double)v[s][j] * exact);
        factor = 1.0f;
    }
#pragma unroll
    for (int s = 0; s < kSmallSlots; ++s) {
        const int slot = s * kSmallThreads + threadIdx.x;
        if (slot >= a.items) continue;
        const TensorDev& t = a.t[tensor_of(a, slot)];
        const long long at = 4ll * (slot - t.first);
        if (t.dtype == LP_F32) store_slot<float>(t, at, v[s], factor);
        else if (t.dtype == LP_BF16) store_slot<__bf16>(t, at, v[s], factor);
        else store_slot<_Float16>(t, at, v[s], factor);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

int dtype_bytes(int t) { return t == LP_F32 ? 4 : 2; }

// How a call is divided.
struct Division {
    bool small;
    bool past_cache;
    long long chunk, items;   // values of a part; parts of all tensors
    size_t bytes;
};

// Parts for 32 workgroups a compute unit, in whole blocks of kLeast values (so that a part starts as its tensor is aligned).
lp_status divide(const std::vector<lp_gradient>& v, Division* out)
{
    Division& d = *out;
    d = {};
    double total = 0.0, bytes = 0.0;
    long long slots = 0;
    for (const lp_gradient& g : v) {
        total += (double)g.size;
        bytes += (double)g.size * dtype_bytes(g.dtype);
        if (slots <= kSmallThreads * kSmallSlots) slots += (g.size + 3) / 4;
    }
    d.small = v.size() <= kSmallTensors && slots <= kSmallThreads * kSmallSlots;
    if (d.small) return LP_OK;
    std::string err;
    int n_cu = 0;
    if (compute_units(&n_cu, &err)) return fail(LP_ERR_HIP, err);
    d.past_cache = bytes > 256e6;   // the Infinity Cache
    d.chunk = ((long long)(total / (32.0 * n_cu)) + kLeast) / kLeast * kLeast;
    for (const lp_gradient& g : v) d.items += (g.size + d.chunk - 1) / d.chunk;
    if (d.items > 1ll << 30) return fail(LP_ERR_UNSUPPORTED, "too many tensors for one call");
    d.bytes = ((size_t)(d.items + 1) * sizeof(double) + 255) / 256 * 256;
    return LP_OK;
}

lp_status collect(int32_t n, const lp_gradient* grads, bool in, bool out, std::vector<lp_gradient>* v)
{
    if (n < 0) return fail(LP_ERR_INVALID_ARG, "n must be >= 0");
    if (n > 0 && !grads) return fail(LP_ERR_INVALID_ARG, "grads must not be NULL");
    for (int k = 0; k < n; ++k) {
        const lp_gradient& g = grads[k];
        const auto name = [&] { return "grads[" + std::to_string(k) + "]"; };
        if (g.dtype != LP_F32 && g.dtype != LP_BF16 && g.dtype != LP_F16)
            return fail(LP_ERR_INVALID_ARG, name() + ".dtype must be LP_F32, LP_BF16 or LP_F16");
        if (g.size < 0) return fail(LP_ERR_INVALID_ARG, name() + ".size must be >= 0");
        if (g.size > 1ll << 48) return fail(LP_ERR_UNSUPPORTED, name() + ".size is beyond 2^48");
        if (!g.size) continue;
        if ((in && !g.in) || (out && !g.out)) return fail(LP_ERR_INVALID_ARG, name() + " has a NULL tensor");
        if ((in && (uintptr_t)g.in % dtype_bytes(g.dtype)) || (out && (uintptr_t)g.out % dtype_bytes(g.dtype)))
            return fail(LP_ERR_INVALID_ARG, name() + " must be aligned to its elements");
        v->push_back(g);
    }
    return LP_OK;
}

// Whether an out lies over another tensor, the norm, or its own in without being it.
bool overlap(const std::vector<lp_gradient>& v, const float* norm)
{
    struct Range {
        uintptr_t from, end;
        bool written;
    };
    std::vector<Range> ranges;
    ranges.reserve(2 * v.size() + 1);
    ranges.push_back({(uintptr_t)norm, (uintptr_t)norm + sizeof(float), true});
    for (const lp_gradient& g : v) {
        const uintptr_t bytes = (uintptr_t)g.size * dtype_bytes(g.dtype);
        ranges.push_back({(uintptr_t)g.out, (uintptr_t)g.out + bytes, true});
        if (g.in != g.out) ranges.push_back({(uintptr_t)g.in, (uintptr_t)g.in + bytes, false});
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

lp_status launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? LP_OK : fail(LP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

template <int MAX>
Set<MAX> set_of(const std::vector<lp_gradient>& v, size_t first, size_t end, long long per_item, long long chunk, int before)
{
    Set<MAX> a;
    std::memset(&a, 0, sizeof(a));
    a.chunk = chunk;
    a.before = before;
    for (size_t k = first; k < end; ++k) {
        a.t[a.n++] = {v[k].in, v[k].out, (long long)v[k].size, a.items, v[k].dtype};
        a.items += (int)((v[k].size + per_item - 1) / per_item);
    }
    return a;
}

lp_status run(const std::vector<lp_gradient>& v, Clip c, void* workspace, size_t workspace_bytes, hipStream_t s)
{
    Division d;
    const lp_status st = divide(v, &d);
    if (st != LP_OK) return st;
    if (d.bytes && (!workspace || workspace_bytes < d.bytes))
        return fail(LP_ERR_WORKSPACE, "workspace is NULL or smaller than lp_grad_norm_workspace_bytes");
    if (d.bytes && (uintptr_t)workspace % 256) return fail(LP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (d.small) {
        hipLaunchKernelGGL(grad_small_kernel, dim3(1), dim3(kSmallThreads), 0, s, set_of<kSmallTensors>(v, 0, v.size(), 4, 0, 0), c);
        return launched("gradient norm launch");
    }
    double* parts = (double*)workspace;
    std::vector<int> before;   // parts of the sets before each set
    int items = 0;
    for (size_t k = 0; k < v.size(); k += kSetTensors) {
        const size_t end = std::min(v.size(), k + kSetTensors);
        before.push_back(items);
        auto go = [&](const auto& a) {
            hipLaunchKernelGGL(grad_squares_kernel, dim3(a.items), dim3(kThreads), 0, s, a, parts);
            items += a.items;
        };
        if (end - k <= kSmallTensors) go(set_of<kSmallTensors>(v, k, end, d.chunk, d.chunk, items));
        else go(set_of<kSetTensors>(v, k, end, d.chunk, d.chunk, items));
    }
    const bool join = !c.scale || items > kJoinAtOnce;
    if (join) hipLaunchKernelGGL(grad_join_kernel, dim3(1), dim3(kSmallThreads), 0, s, parts, items, c.scale ? parts + items : nullptr, c.norm);
    if (c.scale) {
        const double* sums = join ? parts + items : parts;
        const int n = join ? 1 : items;
        for (size_t set = before.size(); set-- > 0;) {
            const size_t k = set * kSetTensors, end = std::min(v.size(), k + kSetTensors);
            const int write_norm = !join && set == 0;
            auto go = [&](const auto& a) {
                if (d.past_cache) hipLaunchKernelGGL((grad_scale_kernel<true>), dim3(a.items), dim3(kThreads), 0, s, a, sums, n, c, write_norm);
                else hipLaunchKernelGGL((grad_scale_kernel<false>), dim3(a.items), dim3(kThreads), 0, s, a, sums, n, c, write_norm);
            };
            if (end - k <= kSmallTensors) go(set_of<kSmallTensors>(v, k, end, d.chunk, d.chunk, before[set]));
            else go(set_of<kSetTensors>(v, k, end, d.chunk, d.chunk, before[set]));
        }
    }
    return launched("gradient norm launch");
}

}  // namespace

}  // namespace lp

extern "C" {

lp_status lp_grad_norm_workspace_bytes(int32_t n, const lp_gradient* grads, size_t* bytes)
try {
    std::vector<lp_gradient> v;
    lp_status st = lp::collect(n, grads, false, false, &v);
    if (st != LP_OK) return st;
    if (!bytes) return lp::fail(LP_ERR_INVALID_ARG, "bytes must not be NULL");
    lp::Division d;
    if ((st = lp::divide(v, &d)) != LP_OK) return st;
    *bytes = d.bytes;
    return LP_OK;
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_grad_norm(int32_t n, const lp_gradient* grads, float* norm, void* workspace, size_t workspace_bytes, void* stream)
try {
    std::vector<lp_gradient> v;
    const lp_status st = lp::collect(n, grads, true, false, &v);
    if (st != LP_OK) return st;
    if (!norm) return lp::fail(LP_ERR_INVALID_ARG, "norm must not be NULL");
    return lp::run(v, {norm, 0.0f, 0.0f, 0}, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

lp_status lp_clip_grad_norm(int32_t n, const lp_gradient* grads, float max_norm, float eps, float* norm, void* workspace,
                            size_t workspace_bytes, void* stream)
try {
    std::vector<lp_gradient> v;
    const lp_status st = lp::collect(n, grads, true, true, &v);
    if (st != LP_OK) return st;
    if (!norm) return lp::fail(LP_ERR_INVALID_ARG, "norm must not be NULL");
    if (!std::isfinite(max_norm) || max_norm < 0.0f || !std::isfinite(eps) || eps < 0.0f)
        return lp::fail(LP_ERR_INVALID_ARG, "max_norm and eps must be finite and >= 0");
    if (lp::overlap(v, norm))
        return lp::fail(LP_ERR_INVALID_ARG, "an out must not overlap another tensor of the call, the norm or a part of its own in");
    return lp::run(v, {norm, max_norm, eps, 1}, workspace, workspace_bytes, (hipStream_t)stream);
} catch (...) {
    return LP_ERR_HIP;
}

}  // extern "C"
