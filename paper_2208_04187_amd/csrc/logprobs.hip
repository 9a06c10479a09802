// Log probabilities of given tokens for AMD MI355X (gfx950), with the entropy and the most probable alternatives of each row of
// logits, and their gradient.  The softmax itself is never stored: a row keeps its logarithm of the sum and its entropy.
//
//   t_j = (z_j - m) log2 e;  S = sum 2^t;  U = sum t 2^t;   lse = m + ln S;  logp_i = (z_i - m) - ln S;  H = ln S - U / S ln 2
//   ln p = z - lse;    dz = g (delta_t - p) - gh p (ln p + H)
//
// One pass over the logits each.  A thread keeps a running (m, S, U) of its share of a row; shares are joined by
// moving both to the larger m.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;         // a maximum to start from that z - max is never -inf - -inf with
constexpr float kGone = -150.0f;                           // 2^t is zero from here on, and t 2^t may be taken as zero
constexpr int kThreads = 256;
constexpr int kUnroll = 4;                                 // pieces a thread has in flight
constexpr int kBatch = kUnroll * kThreads * kPiece;    // columns of a workgroup's batch

// e^z is taken as 2^(z * kLog2e - r) with r = most * kLog2e rounded: one fused multiplication and the machine's 2^x.  What the rounding of r leaves out, 2^-24 of it, is
// the exponent at the maximum itself; it is put back where the row's sum is known (finish), and kLog2e's own error counts z - most times 1e-8.  Below kHuge r is below
// 2^31 and that exponent within 64: 2^x and sums of it stay in range.  From there on two different binary32 numbers are 64 or more apart (2^30 from the number below it, 128 beyond): a term is 1 at the
// maximum and 0 elsewhere, good to e^-64.
constexpr float kHuge = 0x1p30f;
__device__ __forceinline__ bool huge(float most) { return !(fabsf(most) < kHuge); }
__device__ __forceinline__ float point_of(float most) { return huge(most) ? (most < 0.0f ? -2.0f * kHuge : 2.0f * kHuge) : most * kLog2e; }
__device__ __forceinline__ float exp2_of(float t) { return __builtin_amdgcn_exp2f(t); }

// Part of a row: r belongs to `most`, which is at least the largest logit so far less the margin; S = sum of 2^t, U = sum of t 2^t, t = z * kLog2e - r
struct Share { float most, sum, moment; };
// the share seen from a larger maximum
__device__ __forceinline__ void move(Share& s, float most) {
    float t = s.most == most ? 0.0f : huge(most) ? kGone : fmaxf(point_of(s.most) - point_of(most), kGone);
    const float c = exp2_of(t);
    s.moment = c * __builtin_fmaf(t, s.sum, s.moment);
    s.sum *= c;
    s.most = most;
}
__device__ __forceinline__ Share joined(Share a, Share b) {
    const float most = fmaxf(a.most, b.most);
    move(a, most);
    move(b, most);
    return Share{most, a.sum + b.sum, a.moment + b.moment};
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
    float *logp, *entropy, *lse, *low, *top_logp;           // low: what lse's rounding left out
    int64_t* top_ids;
    Share* shares;                                          // [T][splits], where a row is split
    uint64_t* keys;                                         // [T][splits][top]
    int64_t stride, T, V, ignore;
    int64_t split;                                          // columns of a share (a multiple of 8)
    int64_t first;                                          // share that the launch's first workgroup works on
    int splits, top;
};

template <typename T> __device__ __forceinline__ float element(const T* p);
template <> __device__ __forceinline__ float element(const float* p) { return *p; }
template <> __device__ __forceinline__ float element(const uint16_t* p) { return bf16_value(*p); }

// A row's lse = most + ln in two numbers: a log probability is (z - most) - ln, which a common offset of the logits takes no digits from (rounding lse to one number first does:
// at an offset of 10^4 half of 10^-3).  ln is -inf where every logit is.
struct Lse { float most, ln; };
__device__ __forceinline__ float logp_of(float z, const Lse& l) { return l.ln == -__builtin_inff() ? l.ln : (z - l.most) - l.ln; }

// The row's results from its joined share; id and z: the given token and its logit (any number where it is no token)
__device__ __forceinline__ Lse finish(const LogpArgs& a, int64_t row, const Share& s, int64_t id, float z) {
    const bool empty = s.sum == 0.0f;                       // every logit -inf
    const float ln = logf(s.sum);
    const float left = huge(s.most) ? 0.0f : kLn2 * __builtin_fmaf(-s.most, kLog2e, point_of(s.most));     // r less its exact value
    const Lse lse{s.most, ln + left};
    const float one = empty ? -__builtin_inff() : lse.most + lse.ln;
    a.lse[row] = one;
    if (a.low) {
        const float added = one - lse.most;
        a.low[row] = empty ? 0.0f : (lse.most - (one - added)) + (lse.ln - added);      // exact
    }
    if (a.entropy) {
        const float h = ln - s.moment / s.sum * kLn2;
        a.entropy[row] = empty || h < 0.0f ? 0.0f : h;      // (rounding may leave it just below)
    }
    float logp = 0.0f;
    if (id != a.ignore) {
        if (id < 0 || id >= a.V) logp = __uint_as_float(0x7fc00000u);   // no such token
        else logp = logp_of(z, lse);
    }
    a.logp[row] = logp;
    return lse;
}
template <typename T> __device__ __forceinline__ float logit_of(const LogpArgs& a, int64_t row, int64_t id) {
    return id >= 0 && id < a.V ? element(static_cast<const T*>(a.z) + row * a.stride + id) : 0.0f;
}

// The piece at column c of a row that ends at column `end`, -inf behind it
template <typename T> __device__ __forceinline__ Piece<T> load_logits(const T* row, int c, int end) {
    Piece<T> q;
    if (c + kPiece <= end) q.load(row + c);
    else q.load(row + c, 0, end - c, sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u);
    return q;
}
template <typename T> __device__ __forceinline__ void load_logits(const T* row, int c, int end, float* v) {
    const Piece<T> q = load_logits(row, c, end);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q[i];
}

constexpr int kMostTop = 64;
// NT: threads that share a row, 256 or 64
template <int NT> struct TopLds {
    static constexpr int kCandidates = 4 * NT;
    uint64_t keys[NT == 64 ? NT : NT / 2];
    uint64_t found[kCandidates];
    uint64_t bound;
    uint32_t winners[NT];
    uint32_t count, threads;
};

template <int CTRL> __device__ __forceinline__ uint64_t max_with(uint64_t k) {
    const uint64_t o = (uint64_t)dpp<CTRL>((uint32_t)(k >> 32)) << 32 | dpp<CTRL>((uint32_t)k);
    return o > k ? o : k;
}

// Collects the keys from lds.bound up among the columns of the threads whose first key may reach it (upper).  In any order; lds.count may be more than fit.
template <int NT, typename T> __device__ __forceinline__ void collect(const T* row, int c0, int end, uint64_t upper, TopLds<NT>& lds) {
    const uint64_t bound = lds.bound;
    const float least = bound == 1 ? -__builtin_inff() : value_of(bound);
    if (upper >= bound) lds.winners[atomicAdd(&lds.threads, 1u)] = threadIdx.x;
    __syncthreads();
    const uint32_t steps = (uint32_t)(end - c0 + NT * kPiece - 1) / (NT * kPiece), all = lds.threads * steps;
    for (uint32_t i = threadIdx.x; i < all; i += NT) {
        const uint32_t w = i / steps;
        const int c = c0 + (int)((i - w * steps) * NT + lds.winners[w]) * kPiece;
        if (c >= end) continue;
        float v[8];
        load_logits(row, c, end, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (fmaxf(v[j], -__builtin_inff()) < least || c + j >= end) continue;     // (NaN as -inf)
            const uint64_t k = key_of(v[j], (uint32_t)(c + j));
            if (k < bound) continue;
            const uint32_t at = atomicAdd(&lds.count, 1u);
            if (at < lds.kCandidates) lds.found[at] = k;
        }
    }
    __syncthreads();
}

// The `top` first keys of a row's columns from c0 to end, in order, at out[0..top) (0 where there are fewer).  The calling thread's columns are the pieces
// c0 + (s * NT + thread) * 8, s = 0, 1, ...; `seen` is the largest of them, in the batch at column `where` for the first time.  That bounds its first key from both
// sides, without another look.  The top-th of the lower bounds of all groups of threads bounds the top-th key of all from below: only the
// threads that may reach it are looked at again.  64 groups of four threads let through G ln(G / (G - top)) = 24 keys for twenty, but all for 64: from 24 on
// 128 groups of two (89 for 64; putting them in order takes four times as long).  A key for each of the 256 threads instead: 2048 rows of 50048 with
// twenty keys 77 us, 64 here.  A wavefront's rows go by groups of four threads below six keys, of two below twelve, and by single threads from there on: 16384 x 3000 fp32 (and 65536 x 1000
// bfloat16) with five keys 42.3, 42.4 and 43.5 us (72, 78 and 91), with eleven 52.4, 50.2 and 50.1 (79, 84 and 97), with twenty, for which sixteen groups of four are too few, 59.3 by two and 56.5
// by one (90 and 101): longer rows gain by closer bounds, shorter ones by fewer keys to rank.
template <int NT, typename T>
__device__ __forceinline__ void find_top(const T* row, int c0, int end, int top, float seen, int where, TopLds<NT>& lds, uint64_t* out) {
    const int t = threadIdx.x;
    const bool has = c0 + t * kPiece < end;
    const int last = where + (kUnroll - 1) * NT * kPiece + kPiece - 1;
    const int to = last < end ? last : end - 1;
    uint64_t lower = has ? key_of(seen, (uint32_t)to) : 0;
    const int size = top < (NT == 64 ? 6 : 24) ? 4 : NT == 64 && top >= 12 ? 1 : 2, groups = NT / size;
    if (size > 1) lower = max_with<kXor1>(lower);
    if (size > 2) lower = max_with<kXor2>(lower);
    if (t % size == 0) lds.keys[t / size] = lower;
    if (t == 0) { lds.count = lds.threads = 0; lds.bound = 1; }
    __syncthreads();
    if (t < groups) {
        const uint64_t mine = lds.keys[t];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < groups; ++j) {
            const uint64_t k = lds.keys[j];
            rank += k > mine || (k == mine && j < t);
        }
        if (rank == top - 1) lds.bound = mine ? mine : 1;   // fewer groups than `top` have columns: all of them
    }
    __syncthreads();
    collect(row, c0, end, has ? key_of(seen, (uint32_t)where) : 0, lds);
    if (lds.count > lds.kCandidates) {
        // many equal logits at the bound: the threads' first keys themselves give a closer one
        __syncthreads();
        uint64_t best = 0;
        if (has) {
#pragma unroll 1
            for (int u = 0; u < kUnroll; ++u) {             // the first key lies in the batch that `seen` is from; NaN is -inf there too
                const int c = where + u * (NT * kPiece);
                if (c >= end) break;
                float v[8];
                load_logits(row, c, end, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t k = key_of(v[i], (uint32_t)(c + i));
                    if (k > best && c + i < end) best = k;
                }
            }
        }
        lds.found[t] = best;
        if (t == 0) { lds.count = lds.threads = 0; lds.bound = 1; }
        __syncthreads();
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < NT; ++j) rank += lds.found[j] > best;
        if (best && rank == top - 1) lds.bound = best;
        __syncthreads();
        collect(row, c0, end, best, lds);
    }
    const int n = (int)lds.count;
    if (n <= lds.kCandidates) {
        if (t < top && t >= n) out[t] = 0;
        for (int i = t; i < n; i += NT) {
            const uint64_t k = lds.found[i];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += lds.found[j] > k;
            if (rank < top) out[rank] = k;
        }
    } else {
        // still more than fit (a few threads hold nearly all large logits): one after the other, each the first behind the last one
        uint64_t prior = ~0ull;
        for (int r = 0; r < top; ++r) {
            uint64_t mine = 0;
            for (int c = c0 + t * kPiece; c < end; c += NT * kPiece) {
                float v[8];
                load_logits(row, c, end, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t k = key_of(v[i], (uint32_t)(c + i));
                    if (k < prior && k > mine && c + i < end) mine = k;
                }
            }
            __syncthreads();                                // behind the last round's reads
            lds.found[t] = mine;
            __syncthreads();
            uint64_t first = 0;
#pragma unroll 8
            for (int i = 0; i < NT; ++i) first = lds.found[i] > first ? lds.found[i] : first;
            if (t == 0) out[r] = first;
            prior = first;
        }
    }
}

// The workgroup's shares joined; every thread gets the result.  slots: 3 * (NT / 64)
template <int NT> __device__ __forceinline__ Share over_workgroup(const Share& s, float* slots) {
    constexpr int W = NT / 64;
    Share r = s;
    move(r, __uint_as_float(over_lanes<MaxF, 64>(__float_as_uint(s.most))));
    r.sum = sum_lanes<64>(r.sum);
    r.moment = sum_lanes<64>(r.moment);
    if constexpr (W == 1) return r;
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

// A thread's next logits.  most: the largest so far; s is only moved to it where it lies kMargin above: seldom after the first batch,
// while moving every time would be ten instructions for a batch's 330.
constexpr float kMargin = 8.0f;
template <bool ENTROPY, bool TOP>
__device__ __forceinline__ void add_batch(const float (&v)[kUnroll][8], int c, Share& s, float& most, float& seen, int& where) {
    float m = v[0][0];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = u ? 0 : 1; i < 8; ++i) m = fmaxf(m, v[u][i]);
    if constexpr (TOP) {
        if (m > seen) { seen = m; where = c; }
    }
    most = fmaxf(most, m);
    if (most - s.most > kMargin || huge(most)) move(s, most);
    const float r = point_of(s.most);
    if (!huge(most)) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = __builtin_fmaf(v[u][i], kLog2e, -r), e = exp2_of(t);
                s.sum += e;
                if constexpr (ENTROPY) s.moment = __builtin_fmaf(fmaxf(t, kGone), e, s.moment);
            }
    } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = v[u][i] - most;             // NaN: a NaN, or +inf
                s.sum += d < 0.0f ? 0.0f : d == 0.0f ? 1.0f : d;
            }
    }
}

// A row, or a share of one, per workgroup of NT threads: 32 logits a thread and batch, loaded before the first is used; ten and a half vector operations a logit (the machine's 2^x counts four), two
// thirds of what a bfloat16 row's memory traffic leaves time for.  8192 x 50048 bfloat16: 820 MB in 142 us, 5.8 TB/s, with entropy 148 and twenty alternatives 184; 2048 x 50021
// with entropy 50 us and with five alternatives 58, 3.6 TB/s: its rows, eight a CU, all reach their end at the same time, and start at odd elements (50048: 42 and 51).
template <typename T, bool ENTROPY, bool TOP, int NT>
__global__ __launch_bounds__(NT) void log_probs(LogpArgs a) {
    __shared__ float slots[3 * (NT / 64)];
    __shared__ TopLds<NT> lds;
    __shared__ Lse result;
    __shared__ uint64_t first[TOP ? kMostTop : 1];
    const int64_t item = a.first + blockIdx.x, at = a.splits == 1 ? item : item / a.splits;
    const int part = (int)(item - at * a.splits);
    const T* row = static_cast<const T*>(a.z) + at * a.stride;
    const int c0 = (int)(part * a.split), end = (int)(c0 + a.split < a.V ? c0 + a.split : a.V);
    Share s{kLowest, 0.0f, 0.0f};
    float seen = -__builtin_inff(), most = kLowest;
    int where = c0 + (int)threadIdx.x * kPiece;             // the batch of the thread's largest logit
    for (int b = c0; b < end; b += (kUnroll * NT * kPiece)) {
        const int c = b + (int)threadIdx.x * kPiece;
        Piece<T> q[kUnroll];
        if (b + (kUnroll * NT * kPiece) <= end) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) q[u].load(row + c + u * (NT * kPiece));
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) q[u] = load_logits(row, c + u * (NT * kPiece), end);
        }
        float v[kUnroll][8];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = q[u][i];
        add_batch<ENTROPY, TOP>(v, c, s, most, seen, where);
    }
    const int64_t id = a.ids[at];
    const float z = a.splits == 1 ? logit_of<T>(a, at, id) : 0.0f;
    move(s, most);                                          // to the thread's largest itself
    const Share all = over_workgroup<NT>(s, slots);
    if (a.splits == 1) {
        if (threadIdx.x == 0) result = finish(a, at, all, id, z);
    } else if (threadIdx.x == 0) {
        a.shares[item] = all;
    }
    if constexpr (TOP) {
        find_top(row, c0, end, a.top, seen, where, lds, a.splits == 1 ? first : a.keys + item * a.top);
        if (a.splits == 1) {
            __syncthreads();
            const Lse lse = result;
            if ((int)threadIdx.x < a.top) {
                const uint64_t k = first[threadIdx.x];
                a.top_ids[at * a.top + threadIdx.x] = column_of(k);
                a.top_logp[at * a.top + threadIdx.x] = logp_of(value_of(k), lse);
            }
        }
    }
}

constexpr int kMostKeys = 1024;                             // splits * top

// The shares of a row joined, a workgroup a row and turn.  32 shares with twenty alternatives each 5.8 us (82 where all 640 keys were put in order).
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void join_shares(LogpArgs a) {
    __shared__ float slots[3 * (kThreads / 64)];
    __shared__ uint64_t keys[TOP ? kMostKeys : 1], found[TOP ? kMostKeys : 1], bound;
    __shared__ uint32_t count;
    __shared__ Lse result;
    const int t = threadIdx.x, n = TOP ? a.splits * a.top : 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        // all that is read leaves before the first wait
        const int64_t id = a.ids[row];
        const Share share = t < a.splits ? a.shares[row * a.splits + t] : Share{kLowest, 0.0f, 0.0f};
        uint64_t mine[TOP ? kMostKeys / kThreads : 1];
        if constexpr (TOP) {
#pragma unroll
            for (int j = 0; j < kMostKeys / kThreads; ++j) mine[j] = t + j * kThreads < n ? a.keys[row * n + t + j * kThreads] : 0;
        }
        const float z = logit_of<T>(a, row, id);
        const Share all = over_workgroup<kThreads>(share, slots);
        if (t == 0) result = finish(a, row, all, id, z);
        if constexpr (TOP) {
            // each share's keys are in order: of the first few of every share, `top` or more in all, the top-th bounds the row's top-th from
            // below, and only what reaches the bound is put in order
            const int per = (a.top + a.splits - 1) / a.splits;
#pragma unroll
            for (int j = 0; j < kMostKeys / kThreads; ++j) if (t + j * kThreads < n) keys[t + j * kThreads] = mine[j];
            if (t == 0) { count = 0; bound = 1; }
            __syncthreads();
            const Lse lse = result;
            if (t < a.splits * per) {
                const uint64_t k = keys[t / per * a.top + t % per];
                int rank = 0;
                for (int l = 0; l < a.splits; ++l)
                    for (int j = 0; j < per; ++j) rank += keys[l * a.top + j] > k;
                if (k && rank == a.top - 1) bound = k;
            }
            __syncthreads();
            const uint64_t least = bound;
#pragma unroll
            for (int j = 0; j < kMostKeys / kThreads; ++j)
                if (mine[j] >= least) found[atomicAdd(&count, 1u)] = mine[j];  // any order, put in order below
            __syncthreads();
            const int m = (int)count;
            for (int i = t; i < m; i += kThreads) {
                const uint64_t k = found[i];
                int rank = 0;
#pragma unroll 8
                for (int j = 0; j < m; ++j) rank += found[j] > k;
                if (rank < a.top) {
                    a.top_ids[row * a.top + rank] = column_of(k);
                    a.top_logp[row * a.top + rank] = logp_of(value_of(k), lse);
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
    const float *lse, *low, *entropy, *g, *gh;              // low: may be null
    void* out;
    int64_t stride, out_stride, T, V, ignore;
    int64_t parts, first;                                   // batches of a row; the batch that the launch's first workgroup works on
};

// A batch of a row per workgroup, in units of sixteen bytes (513 x 32003 fp32 31 us in pieces of eight elements, 24 so).  Columns are counted from the 16-byte boundary at or before a row's first element, so that units are aligned in rows of any width too; the row's
// are those from `before` to `end`.  (Not in the forward pass, where it would make a row's last bits depend on where the row lies.)  Bound by memory: 4096 x 131072 bfloat16 2147 MB in 346 us,
// 6.2 TB/s; 513 x 32003 fp32 131 MB in 22 us, 6.0.
template <typename T, bool ENTROPY, bool PAST>
__global__ __launch_bounds__(kThreads) void log_probs_back(LogpBackArgs a) {
    constexpr int N = Unit<T>::kSize, U = kBatch / (kThreads * N);
    const int64_t item = a.first + blockIdx.x, at = item / a.parts;
    const T* row = static_cast<const T*>(a.z) + at * a.stride;
    T* out = static_cast<T*>(a.out) + at * a.out_stride;
    const int before = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T)), end = (int)a.V + before;
    const int b = (int)(item - at * a.parts) * kBatch, c0 = b + (int)threadIdx.x * N;
    row -= before;
    out -= before;
    const bool whole = b >= before && b + kBatch <= end;
    // ln p = (z - lse) - low: the second word keeps what p would lose to the rounding of lse (5e-4 of itself at 10^4), and is zero where none is given
    const float lse = a.lse[at], low = a.low ? a.low[at] : 0.0f, h = ENTROPY ? a.entropy[at] - low : 0.0f, gh = ENTROPY ? a.gh[at] : 0.0f;
    const float low2 = low * kLog2e;
    const int64_t id = a.ids[at];
    const bool empty = lse == -__builtin_inff(), token = id >= 0 && id < a.V && id != a.ignore;
    const int own = token ? (int)id + before : -N;
    const float g = id == a.ignore ? 0.0f : token ? a.g[at] : __uint_as_float(0x7fc00000u);
    Unit<T> q[U];
    if (whole) {
#pragma unroll
        for (int u = 0; u < U; ++u) q[u].template load<PAST>(row + c0 + u * (kThreads * N));
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * (kThreads * N);
            if (c >= before && c + N <= end) q[u].template load<PAST>(row + c);
            else q[u].load(row + c, before - c, end - c);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + u * (kThreads * N);
        if (c >= end) break;
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = q[u][i] - lse, p = exp2_of(__builtin_fmaf(d, kLog2e, -low2));
            v[i] = -p * (ENTROPY ? __builtin_fmaf(gh, fmaxf(d, kGone) + h, g) : g);
        }
        if (own >= c && own < c + N) {
#pragma unroll
            for (int i = 0; i < N; ++i) if (own == c + i) v[i] += g;
        }
        if (empty) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.0f;
        }
        if (whole || (c >= before && c + N <= end)) Unit<T>::template store<PAST>(out + c, v);
        else Unit<T>::store(out + c, v, before - c, end - c);
    }
}

// ------------------------------------------------------------------ host side

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)
constexpr int64_t kMostItems = 1 << 23;                    // workgroups of a launch (which may have 2^32 threads)
constexpr int64_t kMostWorkgroups = 1 << 16;               // of a launch whose workgroups take turns
uint32_t grid_of(int64_t items) { return (uint32_t)(items < kMostWorkgroups ? items : kMostWorkgroups); }

int sizes_ok(int64_t T, int64_t V, int64_t stride) {
    if (T < 0 || V < 1 || stride < 0) return DIVISION_EINVAL;
    const int64_t most = int64_t(1) << 40;
    return T > INT32_MAX || V > INT32_MAX - 64 * kThreads * kPiece || (T > 0 && (V > most / T || stride > most / T)) ? DIVISION_ERANGE : DIVISION_OK;
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

template <typename T, int NT> auto log_probs_kernel(const LogpArgs& a) {
    return a.top ? (a.entropy ? log_probs<T, true, true, NT> : log_probs<T, false, true, NT>)
                 : (a.entropy ? log_probs<T, true, false, NT> : log_probs<T, false, false, NT>);
}
// Short rows are one wavefront's each, whose joins need no barrier and whose end costs a quarter: 65536 x 1000 bfloat16 172 -> 42 us, with five alternatives 309 -> 76; 4096 x 8000 bfloat16 26 -> 19.
// Longer ones keep four busier: 4096 x 8000 fp32 24 -> 26, 1024 x 30000 bfloat16 13.8 -> 16.5; twenty alternatives of 4096 x 8000 fp32 33 -> 42, of 4096 x 5000 bfloat16 27 -> 22.
// More than 24 alternatives want more than 64 threads to bound them.
bool short_row(int64_t V, size_t size, int top) { return top <= 24 && V * (int64_t)size <= (top > 5 ? 12288 : 16384); }
template <typename T> int launch_log_probs(LogpArgs a, hipStream_t st) {
    const bool narrow = a.splits == 1 && short_row(a.V, sizeof(T), a.top);
    void (*kern)(LogpArgs) = narrow ? log_probs_kernel<T, 64>(a) : log_probs_kernel<T, kThreads>(a);
    const uint32_t threads = narrow ? 64 : kThreads;
    for (a.first = 0; a.first < a.T * a.splits; a.first += kMostItems) {
        const int64_t items = a.T * a.splits - a.first;
        hipLaunchKernelGGL(kern, dim3((uint32_t)(items < kMostItems ? items : kMostItems)), dim3(threads), 0, st, a);
        CHECKED(launched());
    }
    if (a.splits == 1) return DIVISION_OK;
    kern = a.top ? join_shares<T, true> : join_shares<T, false>;
    hipLaunchKernelGGL(kern, dim3(grid_of(a.T)), dim3(kThreads), 0, st, a);
    return launched();
}

}  // namespace

extern "C" {

size_t division_log_probs_workspace(int64_t T, int64_t V, int top) {
    if (sizes_ok(T, V, 0) != DIVISION_OK || top < 0 || top > kMostTop || top > V) return 0;
    const Split s = split_of(T, V, top);
    return s.splits == 1 ? 0 : (size_t)T * (size_t)s.splits * ((size_t)top * 8u + sizeof(Share));
}

int division_log_probs_low(const division_logits* n, float* lse_low, void* hip_stream) {
    if (!n || !type_ok(n->dt) || n->top < 0 || n->top > kMostTop || n->top > n->V) return DIVISION_EINVAL;
    CHECKED(sizes_ok(n->T, n->V, n->stride));
    if (n->T == 0) return DIVISION_OK;
    if (!n->logits || !n->ids || !n->logp || !n->lse || (n->top && (!n->top_logp || !n->top_ids))) return DIVISION_EINVAL;
    const size_t need = division_log_probs_workspace(n->T, n->V, n->top);
    if (need && !n->workspace) return DIVISION_EINVAL;
    if (!aligned(n->logits, n->dt == DIVISION_BF16 ? 2 : 4) || !aligned(n->ids, 8) || !aligned(n->logp, 4) || !aligned(n->lse, 4) || !aligned(n->entropy, 4) ||
        !aligned(n->top_logp, 4) || !aligned(n->top_ids, 8) || !aligned(n->workspace, 8) || !aligned(lse_low, 4))
        return DIVISION_EALIGN;
    if (n->workspace_bytes < need) return DIVISION_ESIZE;
    const Split s = split_of(n->T, n->V, n->top);
    LogpArgs a{};
    a.z = n->logits; a.ids = n->ids; a.logp = n->logp; a.entropy = n->entropy; a.lse = n->lse; a.low = lse_low; a.top_logp = n->top_logp; a.top_ids = n->top_ids;
    a.keys = static_cast<uint64_t*>(n->workspace);
    a.shares = reinterpret_cast<Share*>(static_cast<char*>(n->workspace) + (size_t)n->T * s.splits * n->top * 8u);
    a.stride = n->stride; a.T = n->T; a.V = n->V; a.ignore = n->ignore_index; a.split = s.columns; a.splits = s.splits; a.top = n->top;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return n->dt == DIVISION_F32 ? launch_log_probs<float>(a, st) : launch_log_probs<uint16_t>(a, st);
}

int division_log_probs(const division_logits* n, void* hip_stream) { return division_log_probs_low(n, nullptr, hip_stream); }

int division_log_probs_backward_low(const division_logits_back* n, const float* lse_low, void* hip_stream) {
    if (!n || !type_ok(n->dt)) return DIVISION_EINVAL;
    CHECKED(sizes_ok(n->T, n->V, n->stride));
    CHECKED(sizes_ok(n->T, n->V, n->grad_stride));
    if (n->T == 0) return DIVISION_OK;
    if (!n->logits || !n->ids || !n->lse || !n->grad_logp || !n->grad_logits || (n->grad_entropy && !n->entropy)) return DIVISION_EINVAL;
    const size_t e = n->dt == DIVISION_BF16 ? 2 : 4;
    if (!aligned(n->logits, e) || !aligned(n->grad_logits, e) || !aligned(n->ids, 8) || !aligned(n->lse, 4) || !aligned(n->entropy, 4) || !aligned(n->grad_logp, 4) ||
        !aligned(n->grad_entropy, 4) || !aligned(lse_low, 4))
        return DIVISION_EALIGN;
    if (n->T > 1 && n->grad_stride < n->V) return DIVISION_EINVAL;          // rows of the gradient must not overlap
    LogpBackArgs a{};
    a.z = n->logits; a.ids = n->ids; a.lse = n->lse; a.low = lse_low; a.entropy = n->entropy; a.g = n->grad_logp; a.gh = n->grad_entropy; a.out = n->grad_logits;
    a.stride = n->stride; a.out_stride = n->grad_stride; a.T = n->T; a.V = n->V; a.ignore = n->ignore_index;
    a.parts = (n->V + kPiece - 1 + kBatch - 1) / kBatch;                    // with the columns before a row's first
    // 4096 x 131072 bfloat16: 374 us through the caches, 347 past them; 2048 x 50048 fp32 174 and 156
    const bool past = 2 * n->T * n->V * (int64_t)e > kCached;
    void (*kern)(LogpBackArgs) = n->dt == DIVISION_F32
        ? (past ? (a.gh ? log_probs_back<float, true, true> : log_probs_back<float, false, true>) : (a.gh ? log_probs_back<float, true, false> : log_probs_back<float, false, false>))
        : (past ? (a.gh ? log_probs_back<uint16_t, true, true> : log_probs_back<uint16_t, false, true>)
                : (a.gh ? log_probs_back<uint16_t, true, false> : log_probs_back<uint16_t, false, false>));
    for (a.first = 0; a.first < a.T * a.parts; a.first += kMostItems) {
        const int64_t items = a.T * a.parts - a.first;
        hipLaunchKernelGGL(kern, dim3((uint32_t)(items < kMostItems ? items : kMostItems)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), a);
        CHECKED(launched());
    }
    return DIVISION_OK;
}

int division_log_probs_backward(const division_logits_back* n, void* hip_stream) { return division_log_probs_backward_low(n, nullptr, hip_stream); }

}  // extern "C"
