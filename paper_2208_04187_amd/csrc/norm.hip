// Root-mean-square norm of token vectors for AMD MI355X (gfx950): forward with the residual's addition and an output in
// 8 bits, the codes' values, backward.
//
//   s = x + residual;  rstd = (mean(s^2) + eps)^(-1/2);  y = s * rstd * w
//   group of y:  a = max|y|;  scale = a / Q;  code = nearest(y * Q / a)          (Q = 127: int8, 448: e4m3)
//   u = dy * w;  n = s * rstd;  dx = rstd * (u - n * mean(u * n)) + dsum;  dw = sum over rows of dy * n
//
// Every kernel is bound by what it reads and writes (ten operations an element).  A row is held in the registers of the threads that share it, so it is read
// once; sums, statistics and scales are fp32, and each result is rounded once, as it is stored.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"

constexpr float kTiny = 0x1p-90f;                          // a group whose largest value is smaller is held as zeros

struct NormArgs {
    const void *x, *residual;
    const void* weight;
    void *sum, *y;
    float* rstd;
    uint8_t* codes;
    float* scales;
    int64_t x_stride, residual_stride, T, D;
    int64_t groups;                                         // scales of a row
    float eps;
    int code, group, shift;                                 // division_code; columns a scale (1 << shift), 0 = the row's
    int weight_bf16;
};

// N columns of the weight, whichever type it has
template <int N, typename C> __device__ __forceinline__ void load_weight(const void* weight, int is_bf16, C c, C D, float* w) {
    if (is_bf16) {
        const auto q = load_some<Some<uint16_t, N>>(static_cast<const uint16_t*>(weight), c, D);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = q[i];
    } else {
        const auto q = load_some<Some<float, N>>(static_cast<const float*>(weight), c, D);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = q[i];
    }
}

// The codes of N values (4 or 8) of a group whose largest has these bits (without its sign).  A group that is not finite has scale NaN and
// codes 0, one of next to nothing scale 0 and codes 0.
template <int N> struct Coded { uint32_t w[N / 4]; float scale; };
template <int N> __device__ __forceinline__ Coded<N> code_of(const float* v, uint32_t most_bits, int code) {
    const float most = __uint_as_float(most_bits);
    const bool finite = most_bits < 0x7f800000u, held = finite && most >= kTiny;
    const float top = code == DIVISION_CODE_INT8 ? 127.0f : 448.0f;
    const float inverse = top / most;
    Coded<N> r;
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const float* e = v + 4 * k;
        if (code == DIVISION_CODE_INT8) {
            // rounded to nearest even by the addition of 1.5 * 2^23, whose last byte then holds the code
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(__builtin_fmaf(e[i], inverse, 12582912.0f)) & 0xffu;
            r.w[k] = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
        } else {
            int q = __builtin_amdgcn_cvt_pk_fp8_f32(e[0] * inverse, e[1] * inverse, 0, false);
            r.w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e[2] * inverse, e[3] * inverse, q, true);
        }
        if (!held) r.w[k] = 0;
    }
    r.scale = !finite ? __uint_as_float(0x7fc00000u) : held ? most / top : 0.0f;
    return r;
}
template <int N, typename C> __device__ __forceinline__ void store_codes(uint8_t* row, C c, C D, const Coded<N>& k) {
    if (c + N <= D) {
        __builtin_memcpy(row + c, k.w, N);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) if (c + i < D) row[c + i] = (uint8_t)(k.w[i / 4] >> (i % 4 * 8));
    }
}
template <int N> __device__ __forceinline__ uint32_t most_of(const float* v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = MaxU::of(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}
// the largest of a group of 32, 64 or 128 columns: N of them in each of as many neighbouring lanes as it takes
template <int N> __device__ __forceinline__ uint32_t most_of_group(uint32_t m, int group) {
    m = over_lanes<MaxU, 32 / N>(m);
    if constexpr (N == 8) {
        if (group >= 64) m = MaxU::of(m, dpp<kHalfMirror>(m));
        if (group >= 128) m = MaxU::of(m, dpp<kMirror>(m));
    } else {
        if (group >= 64) m = MaxU::of(m, dpp<kMirror>(m));
        if (group >= 128) m = MaxU::of(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    }
    return m;
}

// the scale of the group that starts with column c
template <typename C> __device__ __forceinline__ void store_scale(const NormArgs& a, int64_t row, C c, C D, float scale) {
    if (a.group == 0 ? c == 0 : c < D && (c & (a.group - 1)) == 0) a.scales[row * a.groups + (a.group ? c >> a.shift : 0)] = scale;
}

// s of the unit at column c
template <typename T, bool RES, bool PAST, typename C> __device__ __forceinline__ void load_sum(const NormArgs& a, int64_t row, C c, C D, float* v) {
    const auto q = load_some<Unit<T>, PAST>(static_cast<const T*>(a.x) + row * a.x_stride, c, D);
    if constexpr (RES) {
        const auto p = load_some<Unit<T>, PAST>(static_cast<const T*>(a.residual) + row * a.residual_stride, c, D);
#pragma unroll
        for (int i = 0; i < Unit<T>::kSize; ++i) v[i] = q[i] + p[i];
    } else {
#pragma unroll
        for (int i = 0; i < Unit<T>::kSize; ++i) v[i] = q[i];
    }
}

// A row per NT threads, R units of sixteen bytes each: NT * R units hold a row.  The weight stays in registers over all rows of a workgroup; a row waits once for its sum of
// squares (and for its largest value, where one scale is the row's).  16384 x 4096 bfloat16 with the residual and e4m3 codes: 605 MB in 104 us, 5.8 TB/s (a
// large copy: 5.1); 8192 x 4096 fp32 with the residual 5.8 TB/s; 16384 x 768 bfloat16 with the residual, half of it in the last-level cache, 17 us; one row of 4096 3.7 us, which is the start of a
// kernel and two trips to memory.
template <typename T, int NT, int R, bool RES, bool PAST>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_rows(NormArgs a) {
    constexpr int ROWS = NT < 256 ? 256 / NT : 1, N = Unit<T>::kSize;
    __shared__ uint32_t slots[NT > 64 ? 3 * (NT / 64) : 1];
    const int lane = threadIdx.x % NT, D = (int)a.D;
    float w[R][N];
    int turn = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) load_weight<N>(a.weight, a.weight_bf16, (r * NT + lane) * N, D, w[r]);
    for (int64_t row = (int64_t)blockIdx.x * ROWS + row_of_thread<NT>(); row < a.T; row += (int64_t)gridDim.x * ROWS) {
        float v[R][N], sq = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) load_sum<T, RES, PAST>(a, row, (r * NT + lane) * N, D, v[r]);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < N; ++i) sq = __builtin_fmaf(v[r][i], v[r][i], sq);
        sq = row_sum<NT>(sq, slots + turn);
        if constexpr (NT > 64) turn ^= NT / 64;
        const float rstd = 1.0f / sqrtf(sq / (float)a.D + a.eps);
        if (lane == 0 && a.rstd) a.rstd[row] = rstd;
        uint32_t most = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * NT + lane) * N;
            if constexpr (RES) store_some<Unit<T>, PAST>(static_cast<T*>(a.sum) + row * a.D, c, D, v[r]);
#pragma unroll
            for (int i = 0; i < N; ++i) v[r][i] = v[r][i] * rstd * w[r][i];
            if (a.y) store_some<Unit<T>, PAST>(static_cast<T*>(a.y) + row * a.D, c, D, v[r]);
            most = MaxU::of(most, most_of<N>(v[r]));
        }
        if (a.code == DIVISION_CODE_NONE) continue;
        if (a.group == 0) most = over_row<MaxU, NT>(most, slots + (NT > 64 ? 2 * (NT / 64) : 0));
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * NT + lane) * N;
            const Coded<N> k = code_of<N>(v[r], a.group == 0 ? most : most_of_group<N>(most_of<N>(v[r]), a.group), a.code);
            store_codes(a.codes + row * a.D, c, D, k);
            store_scale(a, row, c, D, k.scale);
        }
    }
}

// Rows too long for the registers: read twice (the second time from the caches where they hold it), and a third time where one scale is the row's: the largest |y| is that of y itself,
// as in norm_rows (|s * w|, which the first pass could find, leaves binary32 where y does not).  4096 x 40000 bfloat16: 161 us a call, 1.25 times what a copy
// of the bytes takes; with int8 codes and their reading back 309 us where groups of 64 columns have scales, 325 where rows have.
template <typename T, bool RES>
__global__ __launch_bounds__(1024) void norm_wide(NormArgs a) {
    constexpr int N = Unit<T>::kSize;
    __shared__ uint32_t slots[2 * 16];
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        float sq = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.D; c += 1024 * N) {
            float v[N];
            load_sum<T, RES, false>(a, row, c, a.D, v);
#pragma unroll
            for (int i = 0; i < N; ++i) sq = __builtin_fmaf(v[i], v[i], sq);
        }
        sq = row_sum<1024>(sq, slots);
        const float rstd = 1.0f / sqrtf(sq / (float)a.D + a.eps);
        if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
        uint32_t most = 0;
        if (a.code != DIVISION_CODE_NONE && a.group == 0) {
            for (int64_t c = (int64_t)threadIdx.x * N; c < a.D; c += 1024 * N) {
                float v[N], w[N];
                load_sum<T, RES, false>(a, row, c, a.D, v);
                load_weight<N>(a.weight, a.weight_bf16, c, a.D, w);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = v[i] * rstd * w[i];
                most = MaxU::of(most, most_of<N>(v));
            }
            most = over_row<MaxU, 1024>(most, slots + 16);
        }
        for (int64_t c0 = 0; c0 < a.D; c0 += 1024 * N) {    // every lane takes part in its group's maximum
            const int64_t c = c0 + (int64_t)threadIdx.x * N;
            float v[N], w[N];
            load_sum<T, RES, false>(a, row, c, a.D, v);
            load_weight<N>(a.weight, a.weight_bf16, c, a.D, w);
            if constexpr (RES) store_some<Unit<T>>(static_cast<T*>(a.sum) + row * a.D, c, a.D, v);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v[i] * rstd * w[i];
            if (a.y) store_some<Unit<T>>(static_cast<T*>(a.y) + row * a.D, c, a.D, v);
            if (a.code == DIVISION_CODE_NONE) continue;
            const Coded<N> k = code_of<N>(v, a.group == 0 ? most : most_of_group<N>(most_of<N>(v), a.group), a.code);
            store_codes(a.codes + row * a.D, c, a.D, k);
            store_scale(a, row, c, a.D, k.scale);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ the codes' values

struct ReadArgs {
    const uint8_t* codes;
    const float* scales;
    void* out;
    int64_t T, D, groups;
    int code, group, shift, lanes;                          // lanes a row: a power of two up to 256
};

// Eight codes a lane and turn, as many lanes a row as it has eights.  16384 x 4096 codes into bfloat16: 201 MB in 30 us, 6.7 TB/s (the codes, just written, partly from the cache).
template <typename T>
__global__ __launch_bounds__(256) void read_codes(ReadArgs a) {
    const int rows = 256 / a.lanes, lane = threadIdx.x & (a.lanes - 1);
    for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / a.lanes; row < a.T; row += (int64_t)gridDim.x * rows) {
        const uint8_t* in = a.codes + row * a.D;
        for (int64_t c = (int64_t)lane * kPiece; c < a.D; c += (int64_t)a.lanes * kPiece) {
            uint32_t q[2] = {0, 0};
            if (c + kPiece <= a.D) __builtin_memcpy(q, in + c, 8);
            else for (int i = 0; c + i < a.D; ++i) q[i / 4] |= (uint32_t)in[c + i] << (i % 4 * 8);
            const float scale = a.scales[row * a.groups + (a.group ? c >> a.shift : 0)];
            float v[8];
            if (a.code == DIVISION_CODE_INT8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(q[i / 4] >> (i % 4 * 8)) * scale;
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true);
                    v[4 * i] = lo.x * scale;
                    v[4 * i + 1] = lo.y * scale;
                    v[4 * i + 2] = hi.x * scale;
                    v[4 * i + 3] = hi.y * scale;
                }
            }
            store_some<Piece<T>>(static_cast<T*>(a.out) + row * a.D, c, a.D, v);
        }
    }
}

// ------------------------------------------------------------------ backward

struct BackArgs {
    const void *grad, *s, *grad_sum;
    const void* weight;
    const float* rstd;
    void* dx;
    float* parts;                                           // [gridDim.x][D]: each workgroup's share of dw
    int64_t grad_stride, s_stride, grad_sum_stride, T, D;
    int weight_bf16;
};

// What a thread reads of a row
template <typename T, int R, bool PAST> struct BackRow {
    static constexpr int N = Unit<T>::kSize;
    Unit<T> grad[R], s[R], extra[R];
    float rstd;
    template <int NT> __device__ __forceinline__ void load(const BackArgs& a, int64_t row, int lane, int D) {
        if (row >= a.T) {
#pragma unroll
            for (int r = 0; r < R; ++r) { grad[r].zero(); s[r].zero(); }
            rstd = 0.0f;
            return;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * NT + lane) * N;
            grad[r] = load_some<Unit<T>, PAST>(static_cast<const T*>(a.grad) + row * a.grad_stride, c, D);
            s[r] = load_some<Unit<T>, PAST>(static_cast<const T*>(a.s) + row * a.s_stride, c, D);
        }
        if (a.grad_sum) {
#pragma unroll
            for (int r = 0; r < R; ++r) extra[r] = load_some<Unit<T>, PAST>(static_cast<const T*>(a.grad_sum) + row * a.grad_sum_stride, (r * NT + lane) * N, D);
        }
        rstd = a.rstd[row];
    }
};

// A row per NT threads as in norm_rows, THREADS / NT rows a workgroup side by side; dw grows in the registers of the thread that owns its columns over all
// rows of the workgroup, whose sums meet in LDS at the end: large workgroups leave few shares to add up.  Where the registers hold it (AHEAD), a
// row is loaded while the one before it is worked on.  16384 x 768 bfloat16 with the residual's gradient: 101 MB in 19 us, 5.3 TB/s; 16384 x 4096 537 MB in 88 us, 6.1;
// 8191 x 2561 fp32 without it 252 MB in 50 us, 5.1 (rows of an odd width start at any element).
template <typename T, int NT, int R, int THREADS, bool AHEAD, bool PAST>
__global__ __launch_bounds__(THREADS) void norm_back_rows(BackArgs a) {
    constexpr int ROWS = THREADS / NT, N = Unit<T>::kSize;
    __shared__ uint32_t slots[NT > 64 ? 2 * (THREADS / 64) : 1];
    __shared__ float shares[ROWS > 1 ? THREADS * N : 1];
    const int lane = threadIdx.x % NT, D = (int)a.D;
    float w[R][N], dw[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        load_weight<N>(a.weight, a.weight_bf16, (r * NT + lane) * N, D, w[r]);
#pragma unroll
        for (int i = 0; i < N; ++i) dw[r][i] = 0.0f;
    }
    int turn = 0;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    BackRow<T, R, PAST> q;
    q.template load<NT>(a, (int64_t)blockIdx.x * ROWS + row_of_thread<NT>(), lane, D);
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < a.T; base += step) {
        const int64_t row = base + row_of_thread<NT>();
        BackRow<T, R, PAST> next;
        if constexpr (AHEAD) next.template load<NT>(a, row + step, lane, D);
        float dot = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float n = q.s[r][i] * q.rstd, g = q.grad[r][i];
                dot = __builtin_fmaf(g * w[r][i], n, dot);
                dw[r][i] = __builtin_fmaf(g, n, dw[r][i]);
            }
        const float along = row_sum<NT>(dot, slots + turn) / (float)a.D;
        if constexpr (NT > 64) turn ^= THREADS / 64;
        if (row < a.T) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float d[N];
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = q.rstd * __builtin_fmaf(-(q.s[r][i] * q.rstd), along, q.grad[r][i] * w[r][i]);
                if (a.grad_sum) {
#pragma unroll
                    for (int i = 0; i < N; ++i) d[i] += q.extra[r][i];
                }
                store_some<Unit<T>, PAST>(static_cast<T*>(a.dx) + row * a.D, (r * NT + lane) * N, D, d);
            }
        }
        if constexpr (AHEAD) q = next;
        else q.template load<NT>(a, row + step, lane, D);
    }
    float* part = a.parts + (int64_t)blockIdx.x * a.D;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if constexpr (ROWS > 1) {                           // the workgroup's rows: added up in their order
            if (r) __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) shares[threadIdx.x / NT * (NT * N) + i * NT + lane] = dw[r][i];
            __syncthreads();
            for (int j = threadIdx.x; j < NT * N; j += THREADS) {
                const int c = (r * NT + j % NT) * N + j / NT;
                float t = 0.0f;
#pragma unroll
                for (int k = 0; k < ROWS; ++k) t += shares[k * (NT * N) + j];
                if (c < D) part[c] = t;
            }
        } else {
            store_some<Some<float, N>>(part, (r * NT + lane) * N, D, dw[r]);
        }
    }
}

// Rows too long for the registers: read twice; a workgroup's share of dw lies in memory, each column a thread's own, and is read and written for every
// row.  4096 x 40000 bfloat16 479 us, 2.5 times what a copy of the bytes takes, with the residual's gradient 555, 2.2 times; such rows are rare.
template <typename T>
__global__ __launch_bounds__(1024) void norm_back_wide(BackArgs a) {
    constexpr int N = Unit<T>::kSize;
    __shared__ uint32_t slots[2 * 16];
    float* part = a.parts + (int64_t)blockIdx.x * a.D;
    int turn = 0;
    bool first = true;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        const float rstd = a.rstd[row];
        const T* grad = static_cast<const T*>(a.grad) + row * a.grad_stride;
        const T* s = static_cast<const T*>(a.s) + row * a.s_stride;
        float dot = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.D; c += 1024 * N) {
            const auto p = load_some<Unit<T>>(grad, c, a.D), q = load_some<Unit<T>>(s, c, a.D);
            float w[N];
            load_weight<N>(a.weight, a.weight_bf16, c, a.D, w);
#pragma unroll
            for (int i = 0; i < N; ++i) dot = __builtin_fmaf(p[i] * w[i], q[i] * rstd, dot);
        }
        const float along = row_sum<1024>(dot, slots + turn) / (float)a.D;
        turn ^= 16;
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.D; c += 1024 * N) {
            const auto p = load_some<Unit<T>>(grad, c, a.D), q = load_some<Unit<T>>(s, c, a.D);
            float w[N], u[N], n[N], dw[N];
            load_weight<N>(a.weight, a.weight_bf16, c, a.D, w);
            Some<float, N> had;
            if (first) had.zero();
            else had = load_some<Some<float, N>>(static_cast<const float*>(part), c, a.D);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                n[i] = q[i] * rstd;
                u[i] = p[i] * w[i];
                dw[i] = __builtin_fmaf(p[i], n[i], had[i]);
            }
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = rstd * __builtin_fmaf(-n[i], along, u[i]);
            if (a.grad_sum) {
                const auto extra = load_some<Unit<T>>(static_cast<const T*>(a.grad_sum) + row * a.grad_sum_stride, c, a.D);
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] += extra[i];
            }
            store_some<Unit<T>>(static_cast<T*>(a.dx) + row * a.D, c, a.D, d);
            store_some<Some<float, N>>(part, c, a.D, dw);
        }
        first = false;
    }
}

// dw: the workgroups' shares added up, 64 columns and 16 runs of shares a workgroup, always in the same order.  256 shares of 768 columns 3.9 us (as long with 16 columns
// and 64 runs): the start of a kernel and a trip to memory.
__global__ __launch_bounds__(1024) void add_shares(const float* parts, int64_t count, int64_t D, void* dw, int is_bf16) {
    __shared__ float runs[16][64];
    const int col = threadIdx.x & 63, run = threadIdx.x >> 6;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < D; c0 += (int64_t)gridDim.x * 64) {
        const int64_t c = c0 + col;
        float t = 0.0f;
        if (c < D) {
#pragma unroll 8
            for (int64_t g = run; g < count; g += 16) t += parts[g * D + c];
        }
        runs[run][col] = t;
        __syncthreads();
        if (run == 0 && c < D) {
#pragma unroll
            for (int i = 1; i < 16; ++i) t += runs[i][col];
            if (is_bf16) static_cast<uint16_t*>(dw)[c] = (uint16_t)bf16_pack2(t, 0.0f);
            else static_cast<float*>(dw)[c] = t;
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host side

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
size_t size_of(division_dtype dt) { return dt == DIVISION_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
// sizes that a call takes: rows and columns in 31 bits, elements (strides counted) in 40
int rows_ok(int64_t T, int64_t D) {
    if (T < 0 || D < 1) return DIVISION_EINVAL;
    return T > INT32_MAX || D > INT32_MAX || (T > 0 && D > (int64_t(1) << 40) / T) ? DIVISION_ERANGE : DIVISION_OK;
}
int stride_ok(int64_t stride, int64_t T) {
    if (stride < 0) return DIVISION_EINVAL;
    return T > 0 && stride > (int64_t(1) << 40) / T ? DIVISION_ERANGE : DIVISION_OK;
}
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)

int shift_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

constexpr int64_t kMostWorkgroups = 2048;

// The forward pass: threads a row and units a thread (M: fp32 has half as many elements in one).  Up to 1024 columns a row is one wavefront's, which needs no barrier; of
// bfloat16 up to 2048 (65536 x 2048 110 -> 91 us, 16384 x 1280 with the residual 38 -> 33; of fp32, with eight units a lane, 1999 x 2048 7.9 -> 9.8).
template <typename T, bool RES, bool PAST> void launch_norm(const NormArgs& a, hipStream_t st) {
    constexpr int M = (int)sizeof(T) / 2, W = M == 1 ? 64 : 256;
    const int64_t D = a.D;
    void (*kern)(NormArgs) = D <= 128 ? norm_rows<T, 16 * M, 1, RES, PAST> : D <= 512 ? norm_rows<T, 64, M, RES, PAST> : D <= 1024 ? norm_rows<T, 64, 2 * M, RES, PAST>
                           : D <= 2048 ? norm_rows<T, W, 256 / W * M, RES, PAST> : D <= 4096 ? norm_rows<T, 256, 2 * M, RES, PAST> : D <= 8192 ? norm_rows<T, 256, 4 * M, RES, PAST>
                           : D <= 16384 ? norm_rows<T, 1024, 2 * M, RES, PAST> : norm_wide<T, RES>;
    if constexpr (sizeof(T) == 2 && (PAST || !RES)) {       // (the others would spill)
        if (D > 16384 && D <= 32768) kern = norm_rows<T, 1024, 4 * M, RES, PAST>;
    }
    const int64_t rows = D <= 128 ? 16 / M : D <= 1024 ? 4 : D <= 2048 ? 256 / W : 1, grid = (a.T + rows - 1) / rows;
    hipLaunchKernelGGL(kern, dim3((uint32_t)(grid < kMostWorkgroups ? grid : kMostWorkgroups)), dim3(D <= 8192 ? 256 : 1024), 0, st, a);
}
// Past the caches where they would not hold the call's tensors: 16384 x 4096 bfloat16 with the residual and int8 codes 118 us through them, 102 past them (backward 99.6 and
// 92.5), 8192 x 4096 fp32 with the residual 99.7 and 92.7 (102.5 and 92.3); of 16384 x 1024 bfloat16, which they hold, 27.7 and 27.8 (24.9 and 26.6).
template <typename T, bool RES> void launch_norm(const NormArgs& a, hipStream_t st) {
    const bool past = (1 + 2 * RES + (a.y != nullptr)) * a.T * a.D * (int64_t)sizeof(T) > kCached;
    past ? launch_norm<T, RES, true>(a, st) : launch_norm<T, RES, false>(a, st);
}

// The backward pass: workgroups of 1024 threads, one a CU, so that few shares of dw are left to add up (16384 x 512 bfloat16: 14.6 us, 17.6 with four
// times as many of 256 threads; 8191 x 2561 fp32 68 either way).  A piece a thread and the next row's loads ahead of the work, except from 513 to 1024 columns, where
// two pieces on one wavefront need no barriers and leave fewer lanes idle (16384 x 768 bfloat16 26.4 -> 20.8 us), and beyond 8192.
constexpr int kBackThreads = 1024;
// rows a workgroup holds side by side: M twice the threads a row of up to 128 columns for fp32
int64_t back_workgroups(int64_t T, int64_t D, int M) {
    const int rows = kBackThreads / (D <= 128 ? 16 * M : D <= 1024 ? 64 : D <= 2048 ? 256 : D <= 4096 ? 512 : 1024);
    const int64_t grid = (T + rows - 1) / rows, most = 256;
    return grid < most ? grid : most;
}

template <typename T, bool PAST> void launch_back(const BackArgs& a, hipStream_t st) {
    constexpr int M = (int)sizeof(T) / 2, K = kBackThreads;
    const int64_t D = a.D;
    void (*kern)(BackArgs) = D <= 128 ? norm_back_rows<T, 16 * M, 1, K, true, PAST> : D <= 512 ? norm_back_rows<T, 64, M, K, true, PAST> : D <= 1024 ? norm_back_rows<T, 64, 2 * M, K, false, PAST>
                           : D <= 2048 ? norm_back_rows<T, 256, M, K, true, PAST> : D <= 4096 ? norm_back_rows<T, 512, M, K, true, PAST> : D <= 8192 ? norm_back_rows<T, 1024, M, K, true, PAST>
                           : D <= 16384 ? norm_back_rows<T, 1024, 2 * M, K, false, PAST> : norm_back_wide<T>;
    hipLaunchKernelGGL(kern, dim3((uint32_t)back_workgroups(a.T, D, M)), dim3(kBackThreads), 0, st, a);
}
template <typename T> void launch_back(const BackArgs& a, hipStream_t st) {
    const bool past = (3 + (a.grad_sum != nullptr)) * a.T * a.D * (int64_t)sizeof(T) > kCached;
    past ? launch_back<T, true>(a, st) : launch_back<T, false>(a, st);
}

}  // namespace

extern "C" {

int division_rms_norm(const division_norm* n, void* hip_stream) {
    if (!n || !type_ok(n->dt) || !type_ok(n->weight_dt) || !(n->eps >= 0.0f)) return DIVISION_EINVAL;
    CHECKED(rows_ok(n->T, n->D));
    const bool coded = n->code != DIVISION_CODE_NONE;
    if (coded && n->code != DIVISION_CODE_INT8 && n->code != DIVISION_CODE_E4M3) return DIVISION_EINVAL;
    if (coded && n->group != 0 && n->group != 32 && n->group != 64 && n->group != 128) return DIVISION_EINVAL;
    if (n->T == 0) return DIVISION_OK;
    if (!n->x || !n->weight || (n->residual && !n->sum) || (coded && (!n->codes || !n->scales))) return DIVISION_EINVAL;
    CHECKED(stride_ok(n->x_stride, n->T));
    if (n->residual) CHECKED(stride_ok(n->residual_stride, n->T));
    const size_t e = size_of(n->dt);
    if (!aligned(n->x, e) || !aligned(n->residual, e) || !aligned(n->sum, e) || !aligned(n->y, e) || !aligned(n->weight, size_of(n->weight_dt)) ||
        !aligned(n->rstd, 4) || !aligned(n->scales, 4))
        return DIVISION_EALIGN;
    NormArgs a{};
    a.x = n->x; a.residual = n->residual; a.weight = n->weight; a.sum = n->sum; a.y = n->y; a.rstd = n->rstd;
    a.codes = static_cast<uint8_t*>(n->codes); a.scales = n->scales;
    a.x_stride = n->x_stride; a.residual_stride = n->residual_stride; a.T = n->T; a.D = n->D;
    a.groups = n->group ? (n->D + n->group - 1) / n->group : 1;
    a.eps = n->eps; a.code = n->code; a.group = n->group; a.shift = shift_of(n->group); a.weight_bf16 = n->weight_dt == DIVISION_BF16;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n->dt == DIVISION_F32) n->residual ? launch_norm<float, true>(a, st) : launch_norm<float, false>(a, st);
    else n->residual ? launch_norm<uint16_t, true>(a, st) : launch_norm<uint16_t, false>(a, st);
    return launched();
}

int division_read_codes(const void* codes, const float* scales, int64_t T, int64_t D, division_code code, int group, division_dtype dt, void* out,
                        void* hip_stream) {
    if (!type_ok(dt) || (code != DIVISION_CODE_INT8 && code != DIVISION_CODE_E4M3) || (group != 0 && group != 32 && group != 64 && group != 128)) return DIVISION_EINVAL;
    CHECKED(rows_ok(T, D));
    if (T == 0) return DIVISION_OK;
    if (!codes || !scales || !out) return DIVISION_EINVAL;
    if (!aligned(scales, 4) || !aligned(out, size_of(dt))) return DIVISION_EALIGN;
    ReadArgs a{};
    a.codes = static_cast<const uint8_t*>(codes); a.scales = scales; a.out = out; a.T = T; a.D = D;
    a.code = code; a.group = group; a.shift = shift_of(group); a.groups = group ? (D + group - 1) / group : 1;
    a.lanes = 1;
    while (a.lanes < 256 && (int64_t)a.lanes * kPiece < D) a.lanes *= 2;
    const int64_t rows = 256 / a.lanes, grid = (T + rows - 1) / rows;
    hipLaunchKernelGGL(dt == DIVISION_F32 ? read_codes<float> : read_codes<uint16_t>, dim3((uint32_t)(grid < 16384 ? grid : 16384)), dim3(256), 0,
                       static_cast<hipStream_t>(hip_stream), a);
    return launched();
}

size_t division_rms_norm_backward_workspace(int64_t T, int64_t D) {
    return rows_ok(T, D) != DIVISION_OK ? 0 : (size_t)back_workgroups(T, D, 2) * (size_t)D * 4u;
}

int division_rms_norm_backward(const division_norm_back* n, void* hip_stream) {
    if (!n || !type_ok(n->dt) || !type_ok(n->weight_dt)) return DIVISION_EINVAL;
    CHECKED(rows_ok(n->T, n->D));
    if (!n->grad_weight || (n->T > 0 && (!n->grad_y || !n->sum || !n->weight || !n->rstd || !n->grad_x || !n->workspace))) return DIVISION_EINVAL;
    CHECKED(stride_ok(n->grad_y_stride, n->T));
    CHECKED(stride_ok(n->sum_stride, n->T));
    if (n->grad_sum) CHECKED(stride_ok(n->grad_sum_stride, n->T));
    const size_t e = size_of(n->dt), we = size_of(n->weight_dt);
    if (!aligned(n->grad_y, e) || !aligned(n->sum, e) || !aligned(n->grad_sum, e) || !aligned(n->grad_x, e) || !aligned(n->weight, we) ||
        !aligned(n->grad_weight, we) || !aligned(n->rstd, 4) || !aligned(n->workspace, 4))
        return DIVISION_EALIGN;
    if (n->workspace_bytes < division_rms_norm_backward_workspace(n->T, n->D)) return DIVISION_ESIZE;
    BackArgs a{};
    a.grad = n->grad_y; a.s = n->sum; a.grad_sum = n->grad_sum; a.weight = n->weight; a.rstd = n->rstd; a.dx = n->grad_x;
    a.parts = static_cast<float*>(n->workspace);
    a.grad_stride = n->grad_y_stride; a.s_stride = n->sum_stride; a.grad_sum_stride = n->grad_sum_stride; a.T = n->T; a.D = n->D;
    a.weight_bf16 = n->weight_dt == DIVISION_BF16;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n->T > 0) {
        if (n->dt == DIVISION_F32) launch_back<float>(a, st);
        else launch_back<uint16_t>(a, st);
        CHECKED(launched());
    }
    const int64_t grid = (n->D + 63) / 64;
    hipLaunchKernelGGL(add_shares, dim3((uint32_t)(grid < 65536 ? grid : 65536)), dim3(1024), 0, st, a.parts, n->T > 0 ? back_workgroups(n->T, n->D, n->dt == DIVISION_F32 ? 2 : 1) : 0, n->D,
                       n->grad_weight, a.weight_bf16);
    return launched();
}

}  // extern "C"
