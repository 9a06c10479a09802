// Log probabilities of given tokens for AMD MI355X (gfx950), with the entropy and the most probable alternatives of each row of
// logits, and their gradient.  The softmax itself is never stored: a row keeps its logarithm of the sum and its entropy.
//
//   d_j = z_j - max z;  S = sum e^d;  U = sum d e^d;   lse = max + ln S;  logp_t = z_t - lse;  H = ln S - U / S
//   p = e^(z - lse);    dz = g (delta_t - p) - gh p (ln p + H)
//
// One pass over the logits each.  A thread keeps the running (max, S, U) of its share of a row; shares are joined by
// rescaling both sums to the larger maximum.  S and U are sums of terms of one sign (U <= 0), so nothing cancels.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;         // a maximum to start from that z - max is never -inf - -inf with
constexpr float kGone = -150.0f;                           // e^d is zero from here on, and d * e^d may be taken as zero
constexpr int kThreads = 256;
constexpr int kUnroll = 4;                                 // pieces a thread has in flight

// e^d, d <= 0: one multiplication and the machine's 2^x
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

struct Share { float most, sum, moment; };                 // of (d, e^d): max z, S, U
__device__ __forceinline__ Share joined(const Share& a, const Share& b) {
    Share r;
    r.most = fmaxf(a.most, b.most);
    const float da = fmaxf(a.most - r.most, kGone), db = fmaxf(b.most - r.most, kGone), ca = exp_of(a.most - r.most), cb = exp_of(b.most - r.most);
    r.sum = a.sum * ca + b.sum * cb;
    r.moment = ca * __builtin_fmaf(da, a.sum, a.moment) + cb * __builtin_fmaf(db, b.sum, b.moment);
    return r;
}

// The order of logits: by value, NaN as -inf, equal ones by the lower column.  Both in one whole number, larger = before; 0 = none.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t column) {
    uint32_t b = __float_as_uint(z + 0.0f);                // -0 counts as +0
    if (z != z) b = 0xff800000u;
    return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - column);
}
__device__ __forceinline__ uint32_t column_of(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}

struct LogpArgs {
    const void* z;
    const int64_t* ids;
    float *logp, *entropy, *lse, *top_logp;
    int64_t* top_ids;
    Share* shares;                                          // [T][splits], where a row is split
    uint64_t* keys;                                         // [T][splits][top]
    int64_t stride, T, V, ignore;
    int64_t split;                                          // columns of a share (a multiple of 8)
    int splits, top;
};

template <typename T> __device__ __forceinline__ float element(const T* p);
template <> __device__ __forceinline__ float element(const float* p) { return *p; }
template <> __device__ __forceinline__ float element(const uint16_t* p) { return bf16_value(*p); }

// The row's results from its joined share
template <typename T> __device__ __forceinline__ float finish(const LogpArgs& a, int64_t row, const Share& s) {
    const bool empty = s.sum == 0.0f;                       // every logit -inf
    const float ln = logf(s.sum);
    const float lse = empty ? -__builtin_inff() : s.most + ln;
    a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = empty ? 0.0f : ln - s.moment / s.sum;
    const int64_t id = a.ids[row];
    float logp = 0.0f;
    if (id != a.ignore) {
        if (id < 0 || id >= a.V) logp = __uint_as_float(0x7fc00000u);   // no such token
        else logp = empty ? -__builtin_inff() : element(static_cast<const T*>(a.z) + row * a.stride + id) - lse;
    }
    a.logp[row] = logp;
    return lse;
}
__device__ __forceinline__ float logp_of_top(float z, float lse) { return lse == -__builtin_inff() ? lse : z - lse; }

// The piece at column c of a row that ends at column `end`, -inf behind it
template <typename T> __device__ __forceinline__ void load_logits(const T* row, int64_t c, int64_t end, float* v) {
    if (c + kPiece <= end) {
        Piece<T> q;
        q.load(row + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < end ? element(row + c + i) : -__builtin_inff();
    }
}

constexpr int kMostTop = 64;
constexpr int kCandidates = 1024;
struct TopLds {
    uint64_t keys[kThreads];
    uint64_t found[kCandidates];
    uint32_t winners[kMostTop];
    uint32_t count;
};

// The `top` first keys of columns [c0, c1) of a row, in order, at out[0..top) (0 where there are fewer).  best: the first key of the calling
// thread's columns, which are the pieces c0 + (s * kThreads + thread) * 8, s = 0, 1, ...: the top-th of those bounds the top-th of all
// from below, so that only the columns of the `top` threads with the first keys are looked at again, and of those only what reaches the bound.
template <typename T>
__device__ void find_top(const T* row, int64_t c0, int64_t c1, int top, uint64_t best, TopLds& lds, uint64_t* out) {
    const int t = threadIdx.x;
    lds.keys[t] = best;
    if (t == 0) lds.count = 0;
    if (t < kMostTop) lds.winners[t] = 0xffffffffu;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < kThreads; ++i) before += lds.keys[i] > best;
    if (best && before < top) lds.winners[before] = (uint32_t)t;
    __syncthreads();
    const uint32_t last = lds.winners[top - 1];
    const uint64_t bound = last == 0xffffffffu ? 1 : lds.keys[last];          // fewer threads than `top` have columns: all of them
    for (int w = t >> 6; w < top; w += kThreads / 64) {
        const uint32_t who = lds.winners[w];
        if (who == 0xffffffffu) break;
        for (int64_t c = c0 + ((int64_t)(t & 63) * kThreads + who) * kPiece; c < c1; c += 64 * kThreads * kPiece) {
            float v[8];
            load_logits(row, c, c1, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t k = key_of(v[i], (uint32_t)(c + i));
                if (k >= bound && c + i < c1) {
                    const uint32_t at = atomicAdd(&lds.count, 1u);             // any order: keys differ, and are put in order below
                    if (at < kCandidates) lds.found[at] = k;
                }
            }
        }
    }
    __syncthreads();
    const int n = (int)lds.count;
    if (n <= kCandidates) {
        if (t < top && t >= n) out[t] = 0;
        for (int i = t; i < n; i += kThreads) {
            const uint64_t k = lds.found[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += lds.found[j] > k;
            if (rank < top) out[rank] = k;
        }
    } else {
        // more than fit (a few threads hold nearly all large logits): one after the other, each the first behind the last one
        uint64_t prior = ~0ull;
        for (int r = 0; r < top; ++r) {
            uint64_t mine = 0;
            for (int64_t c = c0 + (int64_t)t * kPiece; c < c1; c += kThreads * kPiece) {
                float v[8];
                load_logits(row, c, c1, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t k = key_of(v[i], (uint32_t)(c + i));
                    if (k < prior && k > mine && c + i < c1) mine = k;
                }
            }
            __syncthreads();                                // behind the last round's reads
            lds.keys[t] = mine;
            __syncthreads();
            uint64_t first = 0;
            for (int i = 0; i < kThreads; ++i) first = lds.keys[i] > first ? lds.keys[i] : first;
            if (t == 0) out[r] = first;
            prior = first;
        }
    }
}

// The workgroup's shares joined; every thread gets the result.  slots: 3 * (kThreads / 64)
__device__ __forceinline__ Share over_workgroup(const Share& s, float* slots) {
    constexpr int W = kThreads / 64;
    Share r;
    r.most = __uint_as_float(over_lanes<MaxF, 64>(__float_as_uint(s.most)));
    const float c = exp_of(s.most - r.most), d = fmaxf(s.most - r.most, kGone);
    r.sum = sum_lanes<64>(s.sum * c);
    r.moment = sum_lanes<64>(c * __builtin_fmaf(d, s.sum, s.moment));
    if ((threadIdx.x & 63) == 0) {
        const int w = threadIdx.x >> 6;
        slots[w] = r.most; slots[W + w] = r.sum; slots[2 * W + w] = r.moment;
    }
    __syncthreads();
    r = Share{slots[0], slots[W], slots[2 * W]};
#pragma unroll
    for (int i = 1; i < W; ++i) r = joined(r, Share{slots[i], slots[W + i], slots[2 * W + i]});
    return r;
}

// A row, or a share of one, per workgroup and turn.
template <typename T, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kThreads) void log_probs(LogpArgs a) {
    __shared__ float slots[3 * (kThreads / 64)];
    __shared__ TopLds lds;
    __shared__ float result;
    __shared__ uint64_t first[TOP ? kMostTop : 1];
    for (int64_t item = blockIdx.x; item < a.T * a.splits; item += gridDim.x) {
        const int64_t at = item / a.splits;
        const int part = (int)(item - at * a.splits);
        const T* row = static_cast<const T*>(a.z) + at * a.stride;
        const int64_t c0 = part * a.split, c1 = c0 + a.split < a.V ? c0 + a.split : a.V;
        Share s{kLowest, 0.0f, 0.0f};
        float seen = -__builtin_inff();
        int64_t where = c0 + (int64_t)threadIdx.x * kPiece;                    // the batch of the thread's largest logit
        for (int64_t c = c0 + (int64_t)threadIdx.x * kPiece; c < c1; c += kUnroll * kThreads * kPiece) {
            float v[kUnroll][8];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) load_logits(row, c + u * (kThreads * kPiece), c1, v[u]);
            float most = s.most;
            if constexpr (TOP) most = -__builtin_inff();
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, v[u][i]);
            if constexpr (TOP) {
                if (most > seen) { seen = most; where = c; }
                most = fmaxf(most, s.most);
            }
            const float scale = exp_of(s.most - most);
            if constexpr (ENTROPY) s.moment = scale * __builtin_fmaf(fmaxf(s.most - most, kGone), s.sum, s.moment);
            s.sum *= scale;
            s.most = most;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = v[u][i] - most, e = exp_of(d);
                    s.sum += e;
                    if constexpr (ENTROPY) s.moment = __builtin_fmaf(fmaxf(d, kGone), e, s.moment);
                }
        }
        const Share all = over_workgroup(s, slots);
        if (a.splits == 1) {
            if (threadIdx.x == 0) result = finish<T>(a, at, all);
        } else if (threadIdx.x == 0) {
            a.shares[item] = all;
        }
        if constexpr (TOP) {
            uint64_t best = 0;
            if (c0 + (int64_t)threadIdx.x * kPiece < c1) {
                for (int u = 0; u < kUnroll; ++u) {
                    const int64_t c = where + u * (kThreads * kPiece);
                    if (c >= c1) break;
                    float v[8];
                    load_logits(row, c, c1, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint64_t k = key_of(v[i], (uint32_t)(c + i));
                        if (k > best && c + i < c1) best = k;
                    }
                }
            }
            find_top(row, c0, c1, a.top, best, lds, a.splits == 1 ? first : a.keys + item * a.top);
            if (a.splits == 1) {
                __syncthreads();
                const float lse = result;
                if ((int)threadIdx.x < a.top) {
                    const uint64_t k = first[threadIdx.x];
                    a.top_ids[at * a.top + threadIdx.x] = column_of(k);
                    a.top_logp[at * a.top + threadIdx.x] = logp_of_top(value_of(k), lse);
                }
            }
        }
        __syncthreads();                                    // before the next turn's slots
    }
}

constexpr int kMostKeys = 1024;                             // splits * top

// The shares of a row joined, a workgroup a row and turn
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void join_shares(LogpArgs a) {
    __shared__ float slots[3 * (kThreads / 64)];
    __shared__ uint64_t keys[TOP ? kMostKeys : 1];
    __shared__ float result;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        const int t = threadIdx.x;
        const Share all = over_workgroup(t < a.splits ? a.shares[row * a.splits + t] : Share{kLowest, 0.0f, 0.0f}, slots);
        if (t == 0) result = finish<T>(a, row, all);
        if constexpr (TOP) {
            const int n = a.splits * a.top;
            for (int i = t; i < n; i += kThreads) keys[i] = a.keys[row * n + i];
            __syncthreads();
            const float lse = result;
            for (int i = t; i < n; i += kThreads) {
                const uint64_t k = keys[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += keys[j] > k;
                if (k && rank < a.top) {
                    a.top_ids[row * a.top + rank] = column_of(k);
                    a.top_logp[row * a.top + rank] = logp_of_top(value_of(k), lse);
                }
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ gradient

struct LogpBackArgs {
    const void* z;
    const int64_t* ids;
    const float *lse, *entropy, *g, *gh;
    void* out;
    int64_t stride, out_stride, T, V, ignore, parts;        // parts: of a row, kUnroll * kThreads pieces each
};

template <typename T, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void log_probs_back(LogpBackArgs a) {
    for (int64_t item = blockIdx.x; item < a.T * a.parts; item += gridDim.x) {
        const int64_t at = item / a.parts, c0 = (item - at * a.parts) * (kUnroll * kThreads * kPiece) + (int64_t)threadIdx.x * kPiece;
        const T* row = static_cast<const T*>(a.z) + at * a.stride;
        T* out = static_cast<T*>(a.out) + at * a.out_stride;
        const float lse = a.lse[at], h = ENTROPY ? a.entropy[at] : 0.0f, gh = ENTROPY ? a.gh[at] : 0.0f;
        const int64_t id = a.ids[at];
        const bool empty = lse == -__builtin_inff();
        float g = a.g[at];
        if (id == a.ignore) g = 0.0f;
        else if (id < 0 || id >= a.V) g = __uint_as_float(0x7fc00000u);
        Piece<T> q[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) q[u] = load_piece(row, c0 + u * (kThreads * kPiece), a.V);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + u * (kThreads * kPiece);
            if (c >= a.V) break;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = q[u][i] - lse, p = exp_of(d);
                v[i] = -p * (ENTROPY ? __builtin_fmaf(gh, fmaxf(d, kGone) + h, g) : g);
            }
            if (id >= c && id < c + kPiece && id != a.ignore) {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (id == c + i) v[i] += g;
            }
            if (empty) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            }
            store_piece(out, c, a.V, v);
        }
    }
}

// ------------------------------------------------------------------ host side

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)
constexpr int64_t kMostWorkgroups = 1 << 16;
uint32_t grid_of(int64_t items) { return (uint32_t)(items < kMostWorkgroups ? items : kMostWorkgroups); }

int sizes_ok(int64_t T, int64_t V, int64_t stride) {
    if (T < 0 || V < 1 || stride < 0) return DIVISION_EINVAL;
    const int64_t most = int64_t(1) << 40;
    return T > INT32_MAX || V > INT32_MAX - 8 * 8192 || (T > 0 && (V > most / T || stride > most / T)) ? DIVISION_ERANGE : DIVISION_OK;
}

// Shares of a row: few rows leave CUs idle
struct Split { int splits; int64_t columns; };
Split split_of(int64_t T, int64_t V, int top) {
    int64_t n = T > 0 ? (1024 + T - 1) / T : 1;
    const int64_t pieces = (V + kThreads * kPiece - 1) / (kThreads * kPiece);
    if (n > pieces) n = pieces;
    if (n > 64) n = 64;
    if (top > 0 && n > kMostKeys / top) n = kMostKeys / top;
    const int64_t columns = (pieces + n - 1) / n * (kThreads * kPiece);
    return {(int)((V + columns - 1) / columns), columns};
}

template <typename T> void launch_log_probs(const LogpArgs& a, hipStream_t st) {
    void (*kern)(LogpArgs) = a.top ? (a.entropy ? log_probs<T, true, true> : log_probs<T, false, true>)
                                   : (a.entropy ? log_probs<T, true, false> : log_probs<T, false, false>);
    hipLaunchKernelGGL(kern, dim3(grid_of(a.T * a.splits)), dim3(kThreads), 0, st, a);
    if (a.splits == 1) return;
    kern = a.top ? join_shares<T, true> : join_shares<T, false>;
    hipLaunchKernelGGL(kern, dim3(grid_of(a.T)), dim3(kThreads), 0, st, a);
}

}  // namespace

extern "C" {

size_t division_log_probs_workspace(int64_t T, int64_t V, int top) {
    if (sizes_ok(T, V, 0) != DIVISION_OK || top < 0 || top > kMostTop || top > V) return 0;
    const Split s = split_of(T, V, top);
    return s.splits == 1 ? 0 : (size_t)T * (size_t)s.splits * ((size_t)top * 8u + sizeof(Share));
}

int division_log_probs(const division_logits* n, void* hip_stream) {
    if (!n || !type_ok(n->dt) || n->top < 0 || n->top > kMostTop || n->top > n->V) return DIVISION_EINVAL;
    CHECKED(sizes_ok(n->T, n->V, n->stride));
    if (n->T == 0) return DIVISION_OK;
    if (!n->logits || !n->ids || !n->logp || !n->lse || (n->top && (!n->top_logp || !n->top_ids))) return DIVISION_EINVAL;
    const size_t need = division_log_probs_workspace(n->T, n->V, n->top);
    if (need && !n->workspace) return DIVISION_EINVAL;
    if (!aligned(n->logits, n->dt == DIVISION_BF16 ? 2 : 4) || !aligned(n->ids, 8) || !aligned(n->logp, 4) || !aligned(n->lse, 4) || !aligned(n->entropy, 4) ||
        !aligned(n->top_logp, 4) || !aligned(n->top_ids, 8) || !aligned(n->workspace, 8))
        return DIVISION_EALIGN;
    if (n->workspace_bytes < need) return DIVISION_ESIZE;
    const Split s = split_of(n->T, n->V, n->top);
    LogpArgs a{};
    a.z = n->logits; a.ids = n->ids; a.logp = n->logp; a.entropy = n->entropy; a.lse = n->lse; a.top_logp = n->top_logp; a.top_ids = n->top_ids;
    a.keys = static_cast<uint64_t*>(n->workspace);
    a.shares = reinterpret_cast<Share*>(static_cast<char*>(n->workspace) + (size_t)n->T * s.splits * n->top * 8u);
    a.stride = n->stride; a.T = n->T; a.V = n->V; a.ignore = n->ignore_index; a.split = s.columns; a.splits = s.splits; a.top = n->top;
    if (n->dt == DIVISION_F32) launch_log_probs<float>(a, static_cast<hipStream_t>(hip_stream));
    else launch_log_probs<uint16_t>(a, static_cast<hipStream_t>(hip_stream));
    return launched();
}

int division_log_probs_backward(const division_logits_back* n, void* hip_stream) {
    if (!n || !type_ok(n->dt)) return DIVISION_EINVAL;
    CHECKED(sizes_ok(n->T, n->V, n->stride));
    CHECKED(sizes_ok(n->T, n->V, n->grad_stride));
    if (n->T == 0) return DIVISION_OK;
    if (!n->logits || !n->ids || !n->lse || !n->grad_logp || !n->grad_logits || (n->grad_entropy && !n->entropy)) return DIVISION_EINVAL;
    const size_t e = n->dt == DIVISION_BF16 ? 2 : 4;
    if (!aligned(n->logits, e) || !aligned(n->grad_logits, e) || !aligned(n->ids, 8) || !aligned(n->lse, 4) || !aligned(n->entropy, 4) || !aligned(n->grad_logp, 4) ||
        !aligned(n->grad_entropy, 4))
        return DIVISION_EALIGN;
    if (n->T > 1 && n->grad_stride < n->V) return DIVISION_EINVAL;          // rows of the gradient must not overlap
    LogpBackArgs a{};
    a.z = n->logits; a.ids = n->ids; a.lse = n->lse; a.entropy = n->entropy; a.g = n->grad_logp; a.gh = n->grad_entropy; a.out = n->grad_logits;
    a.stride = n->stride; a.out_stride = n->grad_stride; a.T = n->T; a.V = n->V; a.ignore = n->ignore_index;
    a.parts = (n->V + kUnroll * kThreads * kPiece - 1) / (kUnroll * kThreads * kPiece);
    void (*kern)(LogpBackArgs) = n->dt == DIVISION_F32 ? (a.gh ? log_probs_back<float, true> : log_probs_back<float, false>)
                                                      : (a.gh ? log_probs_back<uint16_t, true> : log_probs_back<uint16_t, false>);
    hipLaunchKernelGGL(kern, dim3(grid_of(a.T * a.parts)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), a);
    return launched();
}

}  // extern "C"
