// Dropout whose mask is computed and never stored, with the addition to the residual stream, for AMD MI355X (gfx950).
//
//   y = residual + V (.) x / (1 - p), V element by element that of division_dropout_forward with the same p and seed
//
// The backward pass computes V again: the same call on the gradient.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"
#include "dropout_words.h"

constexpr int kThreads = 256, kUnroll = 2;

struct DropoutArgs {
    const void *x, *residual;
    void* y;
    const uint64_t* seed_at;                                // or null
    int64_t n, begin;                                       // elements, and the launch's first one
    uint64_t seed;
    uint32_t thr;
    float by;
};

// Sixteen bytes of each tensor a lane and access, two of them on their way.  An element's words are those of its number alone, whatever the vectors.  Bound by memory: 16384 x 4096 in bfloat16 with a
// residual 59.7 us = 6.7 TB/s; 1999 x 1155 in fp32 4.2 us, the launch and one trip.
template <typename T, bool ADD, bool PAST> __global__ __launch_bounds__(kThreads) void dropout_add(DropoutArgs a) {
    typedef Unit<T> U;
    const uint64_t seed = (a.seed_at ? *a.seed_at : a.seed) ^ kDropoutStream;
    const uint32_t seed_a = mix32((uint32_t)seed ^ 0x243F6A88u), seed_c = mix32((uint32_t)(seed >> 32) ^ 0x85A308D3u);
    const int64_t first = a.begin + ((int64_t)blockIdx.x * kUnroll * kThreads + threadIdx.x) * U::kSize;
    const T *x = static_cast<const T*>(a.x), *r = static_cast<const T*>(a.residual);
    U q[kUnroll], s[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t e = first + (int64_t)u * kThreads * U::kSize;
        q[u] = load_some<U, PAST>(x, e, a.n);
        if constexpr (ADD) s[u] = load_some<U, PAST>(r, e, a.n);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t e = first + (int64_t)u * kThreads * U::kSize;
        const uint32_t k1 = mix32((uint32_t)(e >> 32) ^ seed_a), k2 = mix32(k1 + seed_c);
        float v[U::kSize];
#pragma unroll
        for (int i = 0; i < U::kSize; i += 2) {
            const uint32_t w = pair_word(k1, k2, ((uint32_t)e >> 1) + i / 2);
            v[i] = (w & 0xffffu) >= a.thr ? q[u][i] * a.by : 0.0f;
            v[i + 1] = (w >> 16) >= a.thr ? q[u][i + 1] * a.by : 0.0f;
        }
        if constexpr (ADD) {
#pragma unroll
            for (int i = 0; i < U::kSize; ++i) v[i] += s[u][i];
        }
        store_some<U, PAST>(static_cast<T*>(a.y), e, a.n, v);
    }
}

#include "launch.h"

constexpr int64_t kMostWorkgroups = int64_t(1) << 23;        // of a launch, which has fewer than 2^32 threads

template <typename T> int run(DropoutArgs& a, hipStream_t st) {
    constexpr int64_t per = (int64_t)kThreads * kUnroll * Unit<T>::kSize;
    if (a.n > (int64_t(1) << 35)) return DIVISION_ERANGE;
    const bool past = a.n * (int64_t)sizeof(T) * (a.residual ? 3 : 2) > kCached;
    void (*kernel)(DropoutArgs) = a.residual ? (past ? dropout_add<T, true, true> : dropout_add<T, true, false>) : past ? dropout_add<T, false, true> : dropout_add<T, false, false>;
    for (a.begin = 0; a.begin < a.n; a.begin += kMostWorkgroups * per) {
        const int64_t left = (a.n - a.begin + per - 1) / per;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)(left < kMostWorkgroups ? left : kMostWorkgroups)), dim3(kThreads), 0, st, a);
        CHECKED(launched());
    }
    return DIVISION_OK;
}

}  // namespace

extern "C" {

int division_dropout_add(const void* x, const void* residual, int64_t n, division_dtype dt, double p, uint64_t seed, const uint64_t* device_seed, void* y, void* hip_stream) {
    if (n < 0 || !type_ok(dt) || !(p >= 0.0 && p <= 1.0)) return DIVISION_EINVAL;
    if (n == 0) return DIVISION_OK;
    if (!x || !y) return DIVISION_EINVAL;
    const size_t es = size_of(dt);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(y, es) || !aligned(device_seed, 8)) return DIVISION_EALIGN;
    DropoutArgs a{};
    a.x = x; a.residual = residual; a.y = y; a.n = n; a.seed = seed; a.seed_at = device_seed;
    const double t = (double)(float)p * 65536.0 + 0.5;             // division_dropout_forward takes p in 32 bits
    a.thr = t >= 65536.0 ? 65536u : (uint32_t)t;
    a.by = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return dt == DIVISION_BF16 ? run<uint16_t>(a, st) : run<float>(a, st);
}

}  // extern "C"
