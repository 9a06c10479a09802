// The norms of queries and keys, head by head, and the rotation by their positions, for AMD MI355X (gfx950).
//
//   u = x / sqrt(mean of x^2 over the head + eps) * weight;   pairs (a, b) of u -> (a cos - b sin, a sin + b cos), angle = position * frequency
//
// The angles are counted in turns in binary64 and taken to the nearest whole turn before a sine of 32 bits sees them: positions up to 2^28 turn as exactly as near ones.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"

constexpr int kThreads = 256;

// Strides in elements.  The first `first` workgroups have the first tensor's heads, the others the second's.
struct Side { const void *x, *weight, *grad; int64_t token, head, grad_token, grad_head; void* y; float* rstd; const float* rstd_in; int weight_bf16; };
struct RotateArgs {
    Side side[2];
    const double* frequencies;
    const int64_t* positions;
    float* parts;
    int64_t T;
    int heads[2], block[2], first, D, pairs, rotated;   // pairs: D / 2, the first `rotated` of them turn; block: tokens a workgroup takes at a time
    float eps;
};

// V pairs of a row from pair p on: v[0 .. V - 1] their first elements, v[V ..] the second ones.  NEXT: partners are neighbours, else half the rotated (or of the other) elements apart.
template <typename T, int V, bool NEXT, bool PAST = false> struct Pairs {
    static __device__ __forceinline__ int second(const RotateArgs& a, int p) { return p < a.rotated ? a.rotated : a.pairs - a.rotated; }
    static __device__ __forceinline__ int first(const RotateArgs& a, int p) { return p < a.rotated ? p : a.rotated + p; }
    // as they come from memory, and their values
    struct Raw { Some<T, V == 1 ? 16 / (int)sizeof(T) : V> q[V == 1 ? 1 : 2]; };
    static __device__ __forceinline__ Raw none() {
        Raw r;
#pragma unroll
        for (auto& q : r.q) q.zero();
        return r;
    }
    static __device__ __forceinline__ void fetch(const T* row, const RotateArgs& a, int p, Raw& r) {
        const T* at = NEXT ? row + 2 * p : row + first(a, p);
        const int apart = NEXT ? V : second(a, p);
        if constexpr (V == 1) {
            r.q[0].w[0] = word(at); r.q[0].w[1] = word(at + apart);
        } else {
            r.q[0].template load<PAST>(at); r.q[1].template load<PAST>(at + apart);
        }
    }
    static __device__ __forceinline__ void values(const Raw& r, float* v) {
        if constexpr (V == 1) {
            v[0] = __uint_as_float(r.q[0].w[0]); v[1] = __uint_as_float(r.q[0].w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if constexpr (NEXT) { v[i] = r.q[2 * i / V][2 * i % V]; v[V + i] = r.q[(2 * i + 1) / V][(2 * i + 1) % V]; }
                else { v[i] = r.q[0][i]; v[V + i] = r.q[1][i]; }
            }
        }
    }
    static __device__ __forceinline__ void load(const T* row, const RotateArgs& a, int p, float* v) {
        Raw r;
        fetch(row, a, p, r);
        values(r, v);
    }
    static __device__ __forceinline__ void store(T* row, const RotateArgs& a, int p, const float* v) {
        if constexpr (V == 1) {
            T* at = NEXT ? row + 2 * p : row + first(a, p);
            put1(at, v[0]); put1(at + (NEXT ? 1 : second(a, p)), v[1]);
        } else if constexpr (NEXT) {
            float w[2 * V];
#pragma unroll
            for (int i = 0; i < V; ++i) { w[2 * i] = v[i]; w[2 * i + 1] = v[V + i]; }
            Some<T, V>::template store<PAST>(row + 2 * p, w); Some<T, V>::template store<PAST>(row + 2 * p + V, w + V);
        } else {
            T* at = row + first(a, p);
            Some<T, V>::template store<PAST>(at, v); Some<T, V>::template store<PAST>(at + second(a, p), v + V);
        }
    }
    static __device__ __forceinline__ uint32_t word(const T* p) {
        if constexpr (sizeof(T) == 4) return __float_as_uint(*p);
        else return (uint32_t)*p << 16;
    }
    static __device__ __forceinline__ void put1(T* p, float v) {
        if constexpr (sizeof(T) == 4) *p = v;
        else *p = bf16_of(v);
    }
};

template <int V, bool NEXT> __device__ __forceinline__ void load_weight(const Side& s, const RotateArgs& a, int p, float* w) {
    if (s.weight_bf16) Pairs<uint16_t, V, NEXT>::load(static_cast<const uint16_t*>(s.weight), a, p, w);
    else Pairs<float, V, NEXT>::load(static_cast<const float*>(s.weight), a, p, w);
}

// cosine and sine of the angles of tokens t0 .. t0 + n - 1, [token][pair]
__device__ __forceinline__ void angles(const RotateArgs& a, int64_t t0, int n, float2* to) {
    for (int e = threadIdx.x; e < n * a.rotated; e += kThreads) {
        const int t = e / a.rotated, p = e - t * a.rotated;
        double turns = (double)a.positions[t0 + t] * a.frequencies[p] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        to[e] = make_float2(c, s);
    }
}

// LANES lanes have a head, U times V pairs each; a workgroup takes `block` tokens at a time, all heads of all of them one behind the other: the angles, whose sines in binary64 turns cost most of the
// arithmetic, are taken once for a token's heads and wait in the local memory.  A lane has both elements of its pairs, so that the norm's sum is the only exchange.  Backward each workgroup keeps its
// share of the weights' gradients in registers over all its tokens.
// Bound by memory: 16384 tokens, 32 and 8 heads of 128 in bfloat16, 59 us = 5.7 TB/s; backward 87 us = 5.8 TB/s and 4.5 us for the shares.
template <typename T, int V, int U, int LANES, bool NEXT, bool BACK, bool PAST> __global__ __launch_bounds__(kThreads) void rotate(RotateArgs a) {
    typedef Pairs<T, V, NEXT, PAST> P;
    extern __shared__ __attribute__((aligned(16))) float2 turned[];
    constexpr int kSlots = kThreads / LANES;
    const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const bool second = (int)blockIdx.x >= a.first;
    const Side s = a.side[second ? 1 : 0];
    const int heads = a.heads[second ? 1 : 0], block = a.block[second ? 1 : 0], workgroup = blockIdx.x - (second ? a.first : 0), workgroups = second ? (int)gridDim.x - a.first : a.first;
    float w[U][2 * V], dw[U][2 * V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int p = (u * LANES + lane) * V;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) w[u][i] = dw[u][i] = 0.0f;
        if (p < a.pairs) load_weight<V, NEXT>(s, a, p, w[u]);
    }
    const float over = 1.0f / (float)a.D;
    for (int64_t t0 = (int64_t)workgroup * block; t0 < a.T; t0 += (int64_t)workgroups * block) {
        const int n = (int)(a.T - t0 < block ? a.T - t0 : block), items = n * heads;
        // every lane goes round as often: the sums over lanes take all of them
        const int rounds = (items + kSlots - 1) / kSlots;
        typename P::Raw next_x[U], next_g[U];
        float next_rstd = 0.0f;
        const auto load = [&](int e) {
            const int t = e / heads, h = e - t * heads;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = (u * LANES + lane) * V;
                next_x[u] = P::none();
                if constexpr (BACK) next_g[u] = P::none();
                if (e < items && p < a.pairs) {
                    P::fetch(static_cast<const T*>(s.x) + (t0 + t) * s.token + (int64_t)h * s.head, a, p, next_x[u]);
                    if constexpr (BACK) P::fetch(static_cast<const T*>(s.grad) + (t0 + t) * s.grad_token + (int64_t)h * s.grad_head, a, p, next_g[u]);
                }
            }
            if constexpr (BACK) next_rstd = e < items ? s.rstd_in[t0 * heads + e] : 0.0f;
        };
        load(slot);                                         // on its way while the angles are taken
        __syncthreads();
        angles(a, t0, n, turned);
        __syncthreads();
        for (int k = 0; k < rounds; ++k) {
            const int e = k * kSlots + slot, t = e / heads;
            if (BACK && k) load(e);
            float x[U][2 * V], g[U][2 * V], rstd = next_rstd;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                P::values(next_x[u], x[u]);
                if constexpr (BACK) P::values(next_g[u], g[u]);
            }
            // on its way while these are turned (66.3 us without, 61.9 so); backward the registers count for more (101.5 and 111)
            if (!BACK && k + 1 < rounds) load(e + kSlots);
            float sum = 0.0f;
            float2 cs[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = (u * LANES + lane) * V;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    cs[u][i] = make_float2(1.0f, 0.0f);
                    if (e < items && p + i < a.rotated) cs[u][i] = turned[t * a.rotated + p + i];
                }
                if constexpr (BACK) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {           // turned back
                        const float ga = g[u][i], gb = g[u][V + i];
                        g[u][i] = __builtin_fmaf(ga, cs[u][i].x, gb * cs[u][i].y);
                        g[u][V + i] = __builtin_fmaf(gb, cs[u][i].x, -(ga * cs[u][i].y));
                    }
                }
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) {
                    if constexpr (BACK) {
                        x[u][i] *= rstd;
                        dw[u][i] = __builtin_fmaf(g[u][i], x[u][i], dw[u][i]);
                        g[u][i] *= w[u][i];
                        sum = __builtin_fmaf(g[u][i], x[u][i], sum);
                    } else {
                        sum = __builtin_fmaf(x[u][i], x[u][i], sum);
                    }
                }
            }
            sum = sum_lanes<LANES>(sum);
            if constexpr (BACK) sum *= over;
            else rstd = 1.0f / sqrtf(sum / (float)a.D + a.eps);
            if (e >= items) continue;
            if (!BACK && lane == 0 && s.rstd) s.rstd[t0 * heads + e] = rstd;
            T* out = static_cast<T*>(s.y) + (t0 * heads + e) * a.D;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = (u * LANES + lane) * V;
                if (p >= a.pairs) continue;
                float y[2 * V];
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) {
                    if constexpr (BACK) y[i] = rstd * __builtin_fmaf(-x[u][i], sum, g[u][i]);
                    else y[i] = x[u][i] * rstd * w[u][i];
                }
                if constexpr (!BACK) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float ya = y[i], yb = y[V + i];
                        y[i] = __builtin_fmaf(ya, cs[u][i].x, -(yb * cs[u][i].y));
                        y[V + i] = __builtin_fmaf(ya, cs[u][i].y, yb * cs[u][i].x);
                    }
                }
                P::store(out, a, p, y);
            }
        }
    }
    if constexpr (BACK) {
        // the workgroup's share of the weight's gradient: lanes of a wavefront that have the same columns, then wavefront by wavefront
        float* sums = reinterpret_cast<float*>(turned);     // [D]
        __syncthreads();
        for (int e = threadIdx.x; e < a.D; e += kThreads) sums[e] = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i)
#pragma unroll
                for (int o = LANES; o < 64; o <<= 1) dw[u][i] += __shfl_xor(dw[u][i], o, 64);
        for (int wave = 0; wave < kThreads / 64; ++wave) {
            __syncthreads();
            if ((int)(threadIdx.x >> 6) != wave || (threadIdx.x & 63) >= LANES) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = (u * LANES + lane) * V;
                if (p >= a.pairs) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = NEXT ? 2 * (p + i) : P::first(a, p) + i, d = NEXT ? c + 1 : c + P::second(a, p);
                    sums[c] += dw[u][i];
                    sums[d] += dw[u][V + i];
                }
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < a.D; e += kThreads) a.parts[(int64_t)blockIdx.x * a.D + e] = sums[e];
    }
}

// The weights' gradients from the workgroups' shares, in a fixed order: 32 columns a workgroup, 32 threads a column
struct AddArgs { const float* parts; void* out[2]; int bf16[2]; int first[2], count[2], D, blocks; };
__global__ __launch_bounds__(1024) void add_weight_parts(AddArgs a) {
    __shared__ float sums[32][33];
    const int k = (int)blockIdx.x >= a.blocks, c = ((int)blockIdx.x - k * a.blocks) * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
    float s = 0.0f;
    if (c < a.D) {
#pragma unroll 8
        for (int r = row; r < a.count[k]; r += 32) s += a.parts[(int64_t)(a.first[k] + r) * a.D + c];
    }
    sums[row][threadIdx.x & 31] = s;
    __syncthreads();
    if (row || c >= a.D) return;
    s = 0.0f;
    for (int r = 0; r < 32; ++r) s += sums[r][threadIdx.x];
    if (a.bf16[k]) static_cast<uint16_t*>(a.out[k])[c] = bf16_of(s);
    else static_cast<float*>(a.out[k])[c] = s;
}

// ------------------------------------------------------------------ host side

#include "launch.h"

constexpr int kMostParts = 1024;                            // workgroups of a backward launch, which leave a share of a weight's gradient each: what the CUs hold at once

// Tokens that a workgroup takes at a time: two rounds of its lanes over their heads for each time the angles are taken, one backward (forward one, two, three, four and eight rounds 64, 60.5, 61.5, 61.8
// and 66 us, backward 93, 98.5, 100, 101.5 and 107), one token where tokens are few.
int block_of(int64_t T, int64_t heads, int slots, bool back) {
    int block = (int)((back ? 1 : 2) * slots / heads);
    if (block > 16) block = 16;
    while (block > 1 && T < 1024 * (int64_t)block) block /= 2;
    return block < 1 ? 1 : block;
}
// workgroups of one tensor: forward one for each block of tokens, backward its share of kMostParts
int grid_of(int64_t T, int64_t heads, int64_t all_heads, int block, bool back) {
    if (T == 0 || heads == 0) return 0;
    const int64_t n = (T + block - 1) / block;
    int64_t most = back ? kMostParts * heads / all_heads : 1 << 20;
    if (most < 1) most = 1;
    return (int)(n > most ? most : n);
}

// the tensors' own sizes; `back`: the gradients', which the forward pass has none of
int check(const division_rotate& a, const division_rotate_back* back) {
    if (!type_ok(a.dt) || a.T < 0 || a.D < 2 || a.D > 512 || a.D % 2 || a.rotated < 0 || a.rotated % 2 || a.rotated > a.D || (a.next != 0 && a.next != 1) || !(a.eps >= 0.0f)) return DIVISION_EINVAL;
    if (a.T > 0x7fffffff) return DIVISION_ERANGE;
    for (int k = 0; k < 2; ++k) {
        if (a.heads[k] < 0 || (k == 0 && a.heads[k] == 0)) return DIVISION_EINVAL;
        if (a.heads[k] == 0) continue;
        if (a.heads[k] > 4096) return DIVISION_ERANGE;
        if (!type_ok(a.weight_dt[k]) || !a.weight[k]) return DIVISION_EINVAL;
        if (!aligned(a.weight[k], size_of(a.weight_dt[k]))) return DIVISION_EALIGN;
        if (a.T == 0) continue;
        const int64_t most = int64_t(1) << 40;
        if (!a.x[k] || a.token_strides[k] < 0 || a.head_strides[k] < 0) return DIVISION_EINVAL;
        if (!aligned(a.x[k], size_of(a.dt))) return DIVISION_EALIGN;
        if (a.token_strides[k] > most / a.T || a.head_strides[k] > most / a.heads[k] || a.T * a.heads[k] > most / a.D) return DIVISION_ERANGE;
        if (!back) {
            if (!a.y[k]) return DIVISION_EINVAL;
            if (!aligned(a.y[k], size_of(a.dt)) || !aligned(a.rstd[k], 4)) return DIVISION_EALIGN;
        } else {
            if (!back->grad_y[k] || !back->rstd[k] || !back->grad_x[k] || back->token_strides[k] < 0 || back->head_strides[k] < 0) return DIVISION_EINVAL;
            if (!aligned(back->grad_y[k], size_of(a.dt)) || !aligned(back->rstd[k], 4) || !aligned(back->grad_x[k], size_of(a.dt))) return DIVISION_EALIGN;
            if (back->token_strides[k] > most / a.T || back->head_strides[k] > most / a.heads[k]) return DIVISION_ERANGE;
        }
    }
    if (a.T > 0 && ((a.rotated && !a.frequencies) || !a.positions)) return DIVISION_EINVAL;
    return aligned(a.frequencies, 8) && aligned(a.positions, 8) ? DIVISION_OK : DIVISION_EALIGN;
}

RotateArgs args_of(const division_rotate& a) {
    RotateArgs r{};
    for (int k = 0; k < 2; ++k) {
        r.side[k].x = a.x[k]; r.side[k].weight = a.weight[k];
        r.side[k].token = a.token_strides[k]; r.side[k].head = a.head_strides[k];
        r.side[k].y = a.y[k]; r.side[k].rstd = a.rstd[k];
        r.side[k].weight_bf16 = a.weight_dt[k] == DIVISION_BF16;
        r.heads[k] = (int)a.heads[k];
    }
    r.frequencies = a.frequencies; r.positions = a.positions;
    r.T = a.T; r.D = (int)a.D; r.pairs = (int)a.D / 2; r.rotated = (int)a.rotated / 2; r.eps = a.eps;
    return r;
}

template <typename T, int V, int U, int LANES, bool BACK> int launch(RotateArgs& a, bool next, hipStream_t st) {
    for (int k = 0; k < 2; ++k) a.block[k] = a.heads[k] ? block_of(a.T, a.heads[k], kThreads / LANES, BACK) : 0;
    a.first = grid_of(a.T, a.heads[0], a.heads[0] + a.heads[1], a.block[0], BACK);
    const uint32_t grid = (uint32_t)(a.first + grid_of(a.T, a.heads[1], a.heads[0] + a.heads[1], a.block[1], BACK));
    const int block = a.block[0] > a.block[1] ? a.block[0] : a.block[1];
    size_t lds = (size_t)block * a.rotated * sizeof(float2);
    if (BACK && lds < (size_t)a.D * 4) lds = (size_t)a.D * 4;
    // Calls whose tensors together are beyond the caches go past them (16384 tokens, 32 and 8 heads of 128 in bfloat16: 70.8 us kept, 66.0 so; backward 116 and 107).  Only whole vectors: single
    // elements count on the caches to join them.
    constexpr bool kPast = V > 1;
    const bool past = kPast && a.T * (a.heads[0] + a.heads[1]) * (BACK ? 3 : 2) * a.D * (int64_t)sizeof(T) > kCached;
    void (*kernel)(RotateArgs) = next ? (past ? rotate<T, V, U, LANES, true, BACK, kPast> : rotate<T, V, U, LANES, true, BACK, false>)
                                      : past ? rotate<T, V, U, LANES, false, BACK, kPast> : rotate<T, V, U, LANES, false, BACK, false>;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), lds, st, a);
    return launched();
}
// Heads whose pairs are whole vectors of sixteen bytes; others element by element
template <typename T, bool BACK> int run(RotateArgs& a, bool next, hipStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    if (a.pairs % V || (!next && a.rotated % V)) return a.pairs <= 64 ? launch<T, 1, 4, 16, BACK>(a, next, st) : launch<T, 1, 4, 64, BACK>(a, next, st);
    const int units = a.pairs / V;
    if (units <= 4) return launch<T, V, 1, 4, BACK>(a, next, st);
    if (units <= 8) return launch<T, V, 1, 8, BACK>(a, next, st);
    if (units <= 16) return launch<T, V, 1, 16, BACK>(a, next, st);
    if (units <= 32) return launch<T, V, 1, 32, BACK>(a, next, st);
    if constexpr (sizeof(T) == 4) return launch<T, V, 1, 64, BACK>(a, next, st);
    return DIVISION_EINVAL;
}

}  // namespace

extern "C" {

int division_head_norm_rotate(const division_rotate* rotate, void* hip_stream) {
    if (!rotate) return DIVISION_EINVAL;
    CHECKED(check(*rotate, nullptr));
    if (rotate->T == 0) return DIVISION_OK;
    RotateArgs a = args_of(*rotate);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return rotate->dt == DIVISION_BF16 ? run<uint16_t, false>(a, rotate->next, st) : run<float, false>(a, rotate->next, st);
}

size_t division_head_norm_rotate_backward_workspace(int64_t T, int64_t D) {
    return T <= 0 || T > 0x7fffffff || D < 2 || D > 512 ? 0 : (size_t)(T < kMostParts ? T + 1 : kMostParts + 1) * D * 4 * 2;
}

int division_head_norm_rotate_backward(const division_rotate* rotate, const division_rotate_back* back, void* hip_stream) {
    if (!rotate || !back) return DIVISION_EINVAL;
    CHECKED(check(*rotate, back));
    const division_rotate& f = *rotate;
    for (int k = 0; k < 2; ++k) {
        if (f.heads[k] && !back->grad_weight[k]) return DIVISION_EINVAL;
        if (f.heads[k] && !aligned(back->grad_weight[k], size_of(f.weight_dt[k]))) return DIVISION_EALIGN;
    }
    const size_t need = division_head_norm_rotate_backward_workspace(f.T, f.D);
    if (need && !back->workspace) return DIVISION_EINVAL;
    if (!aligned(back->workspace, 16)) return DIVISION_EALIGN;
    if (back->workspace_bytes < need) return DIVISION_ESIZE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    AddArgs add{};
    if (f.T > 0) {
        RotateArgs a = args_of(f);
        for (int k = 0; k < 2; ++k) {
            Side& s = a.side[k];
            s.grad = back->grad_y[k]; s.grad_token = back->token_strides[k]; s.grad_head = back->head_strides[k];
            s.rstd_in = back->rstd[k]; s.y = back->grad_x[k];
        }
        a.parts = static_cast<float*>(back->workspace);
        CHECKED((f.dt == DIVISION_BF16 ? run<uint16_t, true>(a, f.next, st) : run<float, true>(a, f.next, st)));
        add.parts = a.parts;
        add.count[0] = add.first[1] = a.first;
        add.count[1] = grid_of(f.T, a.heads[1], a.heads[0] + a.heads[1], a.block[1], true);
    }
    add.D = (int)f.D;
    add.blocks = (int)((f.D + 31) / 32);
    for (int k = 0; k < 2; ++k) { add.out[k] = back->grad_weight[k]; add.bf16[k] = f.weight_dt[k] == DIVISION_BF16; }
    hipLaunchKernelGGL(add_weight_parts, dim3((uint32_t)(add.blocks * (f.heads[1] ? 2 : 1))), dim3(1024), 0, st, add);
    return launched();
}

}  // extern "C"
