// The global norm of many gradients and their clipping, for AMD MI355X (gfx950).
//
//   norm = sqrt(sum over all tensors of g^2);   c = min(1, limit / (norm + 1e-6));   out = c * g
//
// Squares are added up in binary64: any binary32 value has one (none overflows or vanishes), and the sum is good to 1e-15.
// A launch serves as many tensors as its argument block holds; a workgroup works on runs of kRun elements, wherever
// tensors end, always the same ones in the same order, so that the norm's bits do not depend on timing.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
constexpr int kRun = kThreads * kUnroll * kPiece;          // elements of a run: 8192

// The tensors of a launch: their first element and, for the clipping, where they go; the first of their runs, counted through the launch; how many elements
// their last run has, and their types in the bits above.  The argument block of a launch may have 4 KB.
constexpr uint32_t kElements = 0x3fff, kInBf16 = 0x4000, kOutBf16 = 0x8000;
template <int N> struct Sources {
    static constexpr int kMost = N;
    const void* in[N];
    uint32_t first[N];
    uint16_t last[N];
    uint32_t runs;                                          // of all
    int count;
};
template <int N> struct Targets { void* out[N]; };
struct NormArgs { Sources<288> t; double* parts; };
struct ClipArgs { Sources<184> t; Targets<184> to; const double *parts, *factor; float* norm; float limit; int count; };
static_assert(sizeof(NormArgs) <= 4096 && sizeof(ClipArgs) <= 4096, "kernel arguments");

// The tensor of a run: the last one whose first run is not behind it.  The lanes hold the first runs of all tensors, so that a search is one read of the argument block
// and not one for each of its steps, which wait for one another (336 M bfloat16 gradients in 194 tensors 123 us by halving, 112 so; 26 M in 161 12.8 and 10.8).
template <typename S> struct Tensors {
    uint32_t first[(S::kMost + 63) / 64];
    __device__ __forceinline__ explicit Tensors(const S& t) {
#pragma unroll
        for (int j = 0; j < (S::kMost + 63) / 64; ++j) {
            const int i = (int)(threadIdx.x & 63) + 64 * j;
            first[j] = i < t.count ? t.first[i] : 0xffffffffu;
        }
    }
    __device__ __forceinline__ int of(uint32_t run) const {
        int k = -1;
#pragma unroll
        for (int j = 0; j < (S::kMost + 63) / 64; ++j) k += __builtin_popcountll(__ballot(first[j] <= run));
        return k;
    }
};
template <typename S> __device__ __forceinline__ int elements_of(const S& t, uint32_t run, int k) {
    const uint32_t end = k + 1 < t.count ? t.first[k + 1] : t.runs;
    return run + 1 < end ? kRun : (int)(t.last[k] & kElements);
}

template <typename T> __device__ __forceinline__ double squares(const T* p, int n) {
    double s = 0.0;
    Piece<T> q[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) q[u] = load_some<Piece<T>>(p, (u * kThreads + (int)threadIdx.x) * kPiece, n);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double g = (double)q[u][i];
            s = __builtin_fma(g, g, s);
        }
    return s;
}

template <int THREADS> __device__ __forceinline__ double over_workgroup(double v, double* slots) {
#pragma unroll
    for (int m = 32; m > 0; m /= 2) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) v += slots[i];
    return v;
}

// parts[workgroup]: the squares of its runs, added up.  Bound by memory: 336 M bfloat16 gradients 671 MB in 112 us, 6.0 TB/s; of 45 MB (11 M fp32 in 62 tensors) 4.1,
// half of whose 11 us are the kernel's start, two trips to memory and the sum across the workgroup.
__global__ __launch_bounds__(kThreads) void add_squares(NormArgs a) {
    __shared__ double slots[kThreads / 64];
    double s = 0.0;
    const Tensors<decltype(a.t)> tensors(a.t);
    for (uint32_t run = blockIdx.x; run < a.t.runs; run += gridDim.x) {
        const int k = tensors.of(run);
        const int64_t c = (int64_t)(run - a.t.first[k]) * kRun;
        const int n = elements_of(a.t, run, k);
        s += a.t.last[k] & kInBf16 ? squares(static_cast<const uint16_t*>(a.t.in[k]) + c, n) : squares(static_cast<const float*>(a.t.in[k]) + c, n);
    }
    s = over_workgroup<kThreads>(s, slots);
    if (threadIdx.x == 0) a.parts[blockIdx.x] = s;
}

// The factor of the clipping: 0 where the norm is infinite, whatever the limit is
__device__ __forceinline__ double factor_of(double norm, float limit) {
    if (norm == __builtin_inf()) return 0.0;
    const double c = limit / (norm + 1e-6);
    return c > 1.0 ? 1.0 : c;                               // NaN stays
}

// The norm from the parts, and the factor (null: only the norm): 2048 parts 4.9 us
__global__ __launch_bounds__(1024) void join_squares(const double* parts, int64_t count, float limit, float* norm, double* factor) {
    __shared__ double slots[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += 1024) s += parts[i];
    s = over_workgroup<1024>(s, slots);
    if (threadIdx.x == 0) {
        const double n = sqrt(s);
        *norm = (float)n;
        if (factor) *factor = factor_of(n, limit);
    }
}

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const uint16_t* p) { return bf16_value(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = bf16_of(v); }

// A run of n elements.  Four a lane and access, so that the lanes' stores lie next to one another whatever the two types are (eight of fp32 are two stores
// with gaps: 336 M gradients 641 us, 491 with four).  Stores go past the caches, which keep what the first pass has read of the gradients instead: 460 us, and of 25.6 M
// gradients 38 us instead of 46.
// A factor below kSmall may leave binary32's normal range, where its products with large elements do not: those are of binary64.
constexpr double kSmall = 0x1p-100;
template <typename I, typename O> __device__ __forceinline__ void scale(const I* p, O* o, int n, double c) {
    constexpr int U = (int)(kRun / (kThreads * 4));
    const float f = (float)c;
    if (n == kRun) {
        Some<I, 4> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u].load(p + (u * kThreads + threadIdx.x) * 4);
        // (asked behind the loads, which need not wait for the factor: 336 M gradients 456 us, 464 with the question before them)
        const bool small = c < kSmall;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[4];
            if (small) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (float)(q[u][i] * c);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = q[u][i] * f;
            }
            Some<O, 4>::template store<true>(o + (u * kThreads + threadIdx.x) * 4, v);
        }
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += kThreads) put(o + i, c < kSmall ? (float)(value(p + i) * c) : value(p + i) * f);
    }
}

// Every tensor times the factor, a run a workgroup; one that stays where it is under a factor of 1 is not touched.  JOIN: every workgroup adds up the
// parts itself, in the same order, instead of a launch between the two passes.  Bound by memory: 336 M bfloat16 gradients into fp32 2013 MB in 338 us, 6.0 TB/s; in
// place 1342 MB in 201 us, 6.7.
template <bool JOIN>
__global__ __launch_bounds__(kThreads) void scale_all(ClipArgs a) {
    double f;
    if constexpr (JOIN) {
        __shared__ double slots[kThreads / 64];
        double s = 0.0;
        for (int i = threadIdx.x; i < a.count; i += kThreads) s += a.parts[i];
        const double norm = sqrt(over_workgroup<kThreads>(s, slots));
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
        f = factor_of(norm, a.limit);
    } else {
        f = *a.factor;
    }
    const uint32_t run = blockIdx.x;
    const int k = Tensors<decltype(a.t)>(a.t).of(run);
    const void* in = a.t.in[k];
    void* out = a.to.out[k];
    if ((float)f == 1.0f && in == out) return;
    const int64_t c = (int64_t)(run - a.t.first[k]) * kRun;
    const int n = elements_of(a.t, run, k);
    switch (a.t.last[k] & (kInBf16 | kOutBf16)) {
        case 0: scale(static_cast<const float*>(in) + c, static_cast<float*>(out) + c, n, f); break;
        case kInBf16: scale(static_cast<const uint16_t*>(in) + c, static_cast<float*>(out) + c, n, f); break;
        case kOutBf16: scale(static_cast<const float*>(in) + c, static_cast<uint16_t*>(out) + c, n, f); break;
        default: scale(static_cast<const uint16_t*>(in) + c, static_cast<uint16_t*>(out) + c, n, f);
    }
}

// ------------------------------------------------------------------ host side

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)

constexpr uint32_t kMostParts = 2048;                       // workgroups of a launch of add_squares
constexpr uint32_t kMostRuns = 1u << 23;                    // of a launch: 2^31 threads
// Up to so many runs every workgroup of the second pass adds up the parts of the first, which saves a launch (1 M gradients 10.4 -> 8.2 us); of 3200 runs it
// costs as much as it saves, of many more 10 us.
constexpr int64_t kFewRuns = 2048;

int check(int64_t count, const division_gradient* g, bool clip) {
    if (count < 0 || (count > 0 && !g)) return DIVISION_EINVAL;
    for (int64_t i = 0; i < count; ++i) {
        if (!type_ok(g[i].dt) || g[i].n < 0 || (clip && !type_ok(g[i].out_dt))) return DIVISION_EINVAL;
        if (g[i].n > (int64_t(1) << 40)) return DIVISION_ERANGE;
        if (g[i].n == 0) continue;
        if (!g[i].grad || (clip && (!g[i].out || (g[i].out == g[i].grad && g[i].out_dt != g[i].dt)))) return DIVISION_EINVAL;
        if (!aligned(g[i].grad, g[i].dt == DIVISION_BF16 ? 2 : 4) || (clip && !aligned(g[i].out, g[i].out_dt == DIVISION_BF16 ? 2 : 4))) return DIVISION_EALIGN;
    }
    return DIVISION_OK;
}

// The launches of a list: calls f(sources) for each, put(place, gradient, element) for each tensor of it.  Tensors without elements are left out, ones of more runs than a launch
// has take several places.
template <int N, typename P, typename F> int launches(int64_t count, const division_gradient* g, Sources<N>& t, P&& put, F&& f) {
    t.count = 0;
    t.runs = 0;
    for (int64_t i = 0; i < count; ++i) {
        const uint32_t types = (g[i].dt == DIVISION_BF16 ? kInBf16 : 0u) | (g[i].out_dt == DIVISION_BF16 ? kOutBf16 : 0u);
        for (int64_t from = 0; from < g[i].n;) {
            if (t.count == N || t.runs == kMostRuns) {
                CHECKED(f(t));
                t.count = 0;
                t.runs = 0;
            }
            const int64_t left = g[i].n - from, room = (int64_t)(kMostRuns - t.runs) * kRun, n = left < room ? left : room;
            const int k = t.count++;
            t.in[k] = static_cast<const char*>(g[i].grad) + from * (g[i].dt == DIVISION_BF16 ? 2 : 4);
            t.first[k] = t.runs;
            t.last[k] = (uint16_t)(types | (uint32_t)((n - 1) % kRun + 1));
            put(k, g[i], from);
            t.runs += (uint32_t)((n + kRun - 1) / kRun);
            from += n;
        }
    }
    return t.count ? f(t) : DIVISION_OK;
}
uint32_t parts_of(uint32_t runs) { return runs < kMostParts ? runs : kMostParts; }
const auto nothing = [](int, const division_gradient&, int64_t) {};

}  // namespace

extern "C" {

size_t division_grad_norm_workspace(int64_t count, const division_gradient* grads) {
    if (check(count, grads, false) != DIVISION_OK) return 0;
    size_t parts = 0;
    NormArgs a;
    launches(count, grads, a.t, nothing, [&](const auto& t) { parts += parts_of(t.runs); return DIVISION_OK; });
    return 16 + parts * 8;
}

int division_clip_grads(int64_t count, const division_gradient* grads, float limit, int clip, float* norm, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
    CHECKED(check(count, grads, clip != 0));
    if (!norm || !workspace || (clip && !(limit >= 0.0f))) return DIVISION_EINVAL;
    if (!aligned(norm, 4) || !aligned(workspace, 16)) return DIVISION_EALIGN;
    if (workspace_bytes < division_grad_norm_workspace(count, grads)) return DIVISION_ESIZE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    double* factor = static_cast<double*>(workspace);
    double* parts = reinterpret_cast<double*>(static_cast<char*>(workspace) + 16);
    int64_t done = 0, runs = 0, made = 0;
    NormArgs a;
    CHECKED(launches(count, grads, a.t, nothing, [&](const auto& t) {
        a.parts = parts + done;
        const uint32_t grid = parts_of(t.runs);
        hipLaunchKernelGGL(add_squares, dim3(grid), dim3(kThreads), 0, st, a);
        done += grid;
        runs += t.runs;
        ++made;
        return launched();
    }));
    const bool join = clip && made == 1 && runs <= kFewRuns;
    if (!join) {
        hipLaunchKernelGGL(join_squares, dim3(1), dim3(1024), 0, st, parts, done, limit, norm, clip ? factor : nullptr);
        CHECKED(launched());
    }
    if (!clip) return DIVISION_OK;
    ClipArgs b;
    b.parts = parts; b.factor = factor; b.norm = norm; b.limit = limit; b.count = (int)done;
    const auto put = [&](int k, const division_gradient& g, int64_t from) { b.to.out[k] = static_cast<char*>(g.out) + from * (g.out_dt == DIVISION_BF16 ? 2 : 4); };
    return launches(count, grads, b.t, put, [&](const auto& t) {
        hipLaunchKernelGGL(join ? scale_all<true> : scale_all<false>, dim3(t.runs), dim3(kThreads), 0, st, b);
        return launched();
    });
}

}  // extern "C"
