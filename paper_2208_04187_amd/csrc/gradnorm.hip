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
constexpr int64_t kRun = kThreads * kUnroll * kPiece;      // elements of a run: 8192

// The tensors of a launch: their first element, where they go (clipping), their number of elements, and the first of their runs counted
// through the launch
template <int N> struct Table {
    const void* in[N];
    void* out[N];
    int64_t n[N];
    uint32_t first[N];
    uint32_t type[N];                                       // bit 0: in is bfloat16, bit 1: out is
    uint32_t runs;                                          // of all
    int count;
};
constexpr int kTensors = 120;                               // 32 bytes each: within 4 KB of arguments
struct NormArgs { Table<kTensors> t; double* parts; };
struct ClipArgs { Table<kTensors> t; const float* factor; };
static_assert(sizeof(NormArgs) <= 4096 && sizeof(ClipArgs) <= 4096, "kernel arguments");

template <int N> __device__ __forceinline__ int tensor_of(const Table<N>& t, uint32_t run) {
    int lo = 0, hi = t.count;                               // the last tensor whose first run is not behind `run`
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= run) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename T> __device__ __forceinline__ double squares(const T* p, int64_t c, int64_t n) {
    double s = 0.0;
    Piece<T> q[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) q[u] = load_piece(p, c + u * (kThreads * kPiece), n);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double g = (double)q[u][i];
            s = __builtin_fma(g, g, s);
        }
    return s;
}

__device__ __forceinline__ double over_workgroup(double v, double* slots, int waves) {
#pragma unroll
    for (int m = 32; m > 0; m /= 2) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
    for (int i = 1; i < waves; ++i) v += slots[i];
    return v;
}

// parts[workgroup]: the squares of its runs, added up
__global__ __launch_bounds__(kThreads) void add_squares(NormArgs a) {
    __shared__ double slots[kThreads / 64];
    double s = 0.0;
    for (uint32_t run = blockIdx.x; run < a.t.runs; run += gridDim.x) {
        const int k = tensor_of(a.t, run);
        const int64_t c = (int64_t)(run - a.t.first[k]) * kRun + (int64_t)threadIdx.x * kPiece;
        s += a.t.type[k] & 1 ? squares(static_cast<const uint16_t*>(a.t.in[k]), c, a.t.n[k]) : squares(static_cast<const float*>(a.t.in[k]), c, a.t.n[k]);
    }
    s = over_workgroup(s, slots, kThreads / 64);
    if (threadIdx.x == 0) a.parts[blockIdx.x] = s;
}

// The norm from the parts, and the factor of the clipping (null: only the norm)
__global__ __launch_bounds__(1024) void join_squares(const double* parts, int64_t count, float limit, float* norm, float* factor) {
    __shared__ double slots[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += 1024) s += parts[i];
    s = over_workgroup(s, slots, 16);
    if (threadIdx.x == 0) {
        const double n = sqrt(s);
        *norm = (float)n;
        if (factor) {
            // in two factors: the second is 1, or a power of two where the first alone would leave binary32's normal range
            double c = limit / (n + 1e-6);
            c = c > 1.0 ? 1.0 : c;                          // NaN stays
            const bool small = c < 0x1p-100;
            factor[0] = (float)(small ? c * 0x1p126 : c);
            factor[1] = small ? 0x1p-126f : 1.0f;
        }
    }
}

template <typename I, typename O> __device__ __forceinline__ void scale(const I* p, O* o, int64_t c, int64_t n, float f, float power) {
    Piece<I> q[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) q[u] = load_piece(p, c + u * (kThreads * kPiece), n);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = q[u][i] * f * power;
        store_piece(o, c + u * (kThreads * kPiece), n, v);
    }
}

// Every tensor times the factor; one that stays where it is under a factor of 1 is not touched
__global__ __launch_bounds__(kThreads) void scale_all(ClipArgs a) {
    const float f = a.factor[0], power = a.factor[1];
    for (uint32_t run = blockIdx.x; run < a.t.runs; run += gridDim.x) {
        const int k = tensor_of(a.t, run);
        if (f == 1.0f && power == 1.0f && a.t.in[k] == a.t.out[k]) continue;
        const int64_t c = (int64_t)(run - a.t.first[k]) * kRun + (int64_t)threadIdx.x * kPiece, n = a.t.n[k];
        const void* in = a.t.in[k];
        void* out = a.t.out[k];
        switch (a.t.type[k]) {
            case 0: scale(static_cast<const float*>(in), static_cast<float*>(out), c, n, f, power); break;
            case 1: scale(static_cast<const uint16_t*>(in), static_cast<float*>(out), c, n, f, power); break;
            case 2: scale(static_cast<const float*>(in), static_cast<uint16_t*>(out), c, n, f, power); break;
            default: scale(static_cast<const uint16_t*>(in), static_cast<uint16_t*>(out), c, n, f, power);
        }
    }
}

// ------------------------------------------------------------------ host side

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)

constexpr uint32_t kMostWorkgroups = 2048;                  // of a launch
constexpr uint32_t kMostRuns = 1u << 27;                    // of a launch: 2^40 elements

int check(int64_t count, const division_gradient* g, bool clip) {
    if (count < 0 || (count > 0 && !g)) return DIVISION_EINVAL;
    for (int64_t i = 0; i < count; ++i) {
        if (!type_ok(g[i].dt) || g[i].n < 0 || (clip && !type_ok(g[i].out_dt))) return DIVISION_EINVAL;
        if (g[i].n > (int64_t(1) << 40)) return DIVISION_ERANGE;
        if (g[i].n == 0) continue;
        if (!g[i].grad || (clip && !g[i].out)) return DIVISION_EINVAL;
        if (!aligned(g[i].grad, g[i].dt == DIVISION_BF16 ? 2 : 4) || (clip && !aligned(g[i].out, g[i].out_dt == DIVISION_BF16 ? 2 : 4))) return DIVISION_EALIGN;
    }
    return DIVISION_OK;
}

// The launches of a list: calls f(table) for each; tensors without elements are left out
template <typename F> int launches(int64_t count, const division_gradient* g, F&& f) {
    Table<kTensors> t;
    t.count = 0;
    t.runs = 0;
    for (int64_t i = 0; i <= count; ++i) {
        if (i < count && g[i].n == 0) continue;
        const uint32_t runs = i < count ? (uint32_t)((g[i].n + kRun - 1) / kRun) : 0;
        if (t.count > 0 && (i == count || t.count == kTensors || t.runs + runs > kMostRuns)) {
            CHECKED(f(t));
            t.count = 0;
            t.runs = 0;
        }
        if (i == count) break;
        t.in[t.count] = g[i].grad;
        t.out[t.count] = g[i].out;
        t.n[t.count] = g[i].n;
        t.first[t.count] = t.runs;
        t.type[t.count] = (g[i].dt == DIVISION_BF16 ? 1u : 0u) | (g[i].out_dt == DIVISION_BF16 ? 2u : 0u);
        t.runs += runs;
        ++t.count;
    }
    return DIVISION_OK;
}
uint32_t workgroups(uint32_t runs) { return runs < kMostWorkgroups ? runs : kMostWorkgroups; }

}  // namespace

extern "C" {

size_t division_grad_norm_workspace(int64_t count, const division_gradient* grads) {
    if (check(count, grads, false) != DIVISION_OK) return 0;
    size_t parts = 0;
    launches(count, grads, [&](const Table<kTensors>& t) { parts += workgroups(t.runs); return DIVISION_OK; });
    return 16 + parts * 8;
}

int division_clip_grads(int64_t count, const division_gradient* grads, float limit, int clip, float* norm, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
    CHECKED(check(count, grads, clip != 0));
    if (!norm || !workspace || (clip && !(limit >= 0.0f))) return DIVISION_EINVAL;
    if (!aligned(norm, 4) || !aligned(workspace, 16)) return DIVISION_EALIGN;
    if (workspace_bytes < division_grad_norm_workspace(count, grads)) return DIVISION_ESIZE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    float* factor = static_cast<float*>(workspace);
    double* parts = reinterpret_cast<double*>(static_cast<char*>(workspace) + 16);
    int64_t done = 0;
    CHECKED(launches(count, grads, [&](const Table<kTensors>& t) {
        const uint32_t grid = workgroups(t.runs);
        hipLaunchKernelGGL(add_squares, dim3(grid), dim3(kThreads), 0, st, NormArgs{t, parts + done});
        done += grid;
        return launched();
    }));
    hipLaunchKernelGGL(join_squares, dim3(1), dim3(1024), 0, st, parts, done, limit, norm, clip ? factor : nullptr);
    CHECKED(launched());
    if (!clip) return DIVISION_OK;
    return launches(count, grads, [&](const Table<kTensors>& t) {
        hipLaunchKernelGGL(scale_all, dim3(workgroups(t.runs)), dim3(kThreads), 0, st, ClipArgs{t, factor});
        return launched();
    });
}

}  // extern "C"
