// The backward pass of attention for AMD MI355X (gfx950).
//
//   p = exp(scale q k^T - lse),   ds = p (grad v^T - rowsum(grad out)),   dq = scale ds k,   dk = scale ds^T q,   dv = p^T grad
//
// The probabilities are computed again from lse, twice: once by workgroups that own queries (dq), once by ones that own keys (dk and dv, over all query heads that share them).  Seven
// products instead of five, but every sum is in a workgroup's registers, in an order that sizes alone decide.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"
#include "fastdiv.h"
#include "tiles.h"
#include "attention_args.h"

struct BackArgs : AttentionArgs {
    const char *grad, *o;
    Heads gs;
    char *dq, *dk, *dv;
    float *key_sums, *query_sums;                       // the parts of dk and dv, where the columns are cut, and of dq, where the keys are
    int query_splits, least_keys, least_columns;        // parts, and how many tiles one has at least
    float* stats;                                       // [group][column][2]: lse in powers of two (infinity where nothing is seen), rowsum(grad out)
    FastDiv by_R;
};

// a lane's column of blocks [DP][32], times `by`, to a row
template <typename T, int DP> __device__ __forceinline__ void put_column(T* row, const f32x16* o, float by, int D, int half) {
#pragma unroll
    for (int d = 0; d < DP; d += 8) {
        if (d >= D) continue;
        const f32x16& b = o[d / 32];
        const int n = d % 32 / 2;
        put4(row + d + 4 * half, b[n] * by, b[n + 1] * by, b[n + 2] * by, b[n + 3] * by);
    }
}
// a lane's part of a row as the operands of its column; zeros where it is not `there`
template <typename T, int DP> __device__ __forceinline__ void get_column(Operand<T>* v, const char* row, bool there, int row_bytes, int half) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const int at = (16 * s + 8 * half) * (int)sizeof(T);
        v[s] = there && at < row_bytes ? Operand<T>::at(row + at) : Operand<T>::zero();
    }
}

constexpr int kThreads = 256;

// A workgroup's part of the tiles lo .. hi - 1 that it would have to look at: equal parts, of so many tiles at least
__device__ __forceinline__ void part_of(int split, int splits, int least, int& lo, int& hi) {
    if (splits == 1) return;
    const int each = max((hi - lo + splits - 1) / splits, least);
    lo += split * each;
    hi = min(lo + each, hi);
}

// Adds up what SETS sets of THREADS threads each have in their blocks, into the first set's, through the local memory: a set at a time
template <int SETS, int THREADS, int N> __device__ __forceinline__ void add_sets(f32x16* o, char* memory, int set, int thread) {
    f32x4* sums = reinterpret_cast<f32x4*>(memory) + thread;
#pragma unroll
    for (int s = 1; s < SETS; ++s) {
        __syncthreads();
        if (set == s) {
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[(4 * d + e) * THREADS] = f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
        }
        __syncthreads();
        if (set == 0) {
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 more = sums[(4 * d + e) * THREADS];
#pragma unroll
                    for (int f = 0; f < 4; ++f) o[d][4 * e + f] += more[f];
                }
        }
    }
}

// Wavefronts of 32 columns (queries) each, WAVES of them, share the tiles of the keys and values.  SETS such take every SETS-th tile each.  Z = K Q^T and dP = V grad^T have a query a lane, to whom
// its lse and rowsum belong; dS's registers are the operand of dQ = K^T dS as they are.  The rowsum is left in `stats` for the other kernel.
// Three products.  Bound by the matrix unit and its power: 2 x 4096 tokens, 32 heads on 8 of 128 in bfloat16, causal, 392 to 416 us = 990 to 1050 TFLOP/s; 2 x 1531 tokens of 12 heads of 64 in fp32,
// window 256, 87 us, of which the products of whole tiles alone are 56.
template <typename T, int DP, int KT, int WAVES, int SETS> __global__ __launch_bounds__(64 * WAVES * SETS, sizeof(T) == 2 ? 2 : 1) void back_queries(BackArgs a) {
    constexpr int kTile = Tile<T, DP, KT>::kBytes, kSet = 64 * WAVES, kCols = 32 * WAVES;
    static_assert(SETS == 1 || kSet * (DP / 32) * 64 <= 4 * SETS * kTile, "a set's blocks in place of the tiles");
    __shared__ __attribute__((aligned(16))) char memory[SETS * 4 * kTile];
    const int set = SETS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / kSet), thread = threadIdx.x % kSet, lane = thread & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    char* mine = memory + set * 4 * kTile;
    const int group = blockIdx.x % a.groups, split = blockIdx.x / a.groups % a.query_splits, block = a.blocks - 1 - blockIdx.x / a.groups / a.query_splits;
    const int b = group / a.G, g = group % a.G;
    const uint32_t cols = (uint32_t)a.Sq * (uint32_t)a.R, first_col = (uint32_t)block * kCols;
    const uint32_t wave_col = first_col + 32 * wave, col = wave_col + (lane & 31);
    const Seen seen = seen_of(a, b);
    const int first_key = seen.from(0);                     // what stands before every query's keys is not looked at either
    const uint32_t last_col = min(first_col + kCols - 1, cols - 1), wave_last = min(wave_col + 31u, cols - 1);
    int lo = seen.from((int)(first_col / (uint32_t)a.R)) / KT, hi = (seen.to((int)(last_col / (uint32_t)a.R)) + KT - 1) / KT;
    part_of(split, a.query_splits, a.least_keys, lo, hi);
    const bool works = wave_col < cols, there = col < cols;
    const int qa = works ? (int)(wave_col / (uint32_t)a.R) : 0, qb = works ? (int)(wave_last / (uint32_t)a.R) : 0;
    const int whole_from = seen.from(qb), whole_to = seen.to(qa);
    const int i = (int)(min(col, cols - 1) / (uint32_t)a.R), r = (int)(min(col, cols - 1) % (uint32_t)a.R);
    const int from = seen.from(i), to = there ? max(from, seen.to(i)) : from;
    const char* k = a.k + b * a.ks.batch + (int64_t)g * a.ks.head;
    const char* v = a.v + b * a.vs.batch + (int64_t)g * a.vs.head;
    const int row_bytes = a.D * (int)sizeof(T);
    const auto fetch = [&](int t, int at) {
        const int low = first_key - t * KT, left = seen.keys - t * KT;
        char* to = mine + at * 2 * kTile;
        Tile<T, DP, KT>::template fill<kSet>(to, k + (int64_t)t * KT * a.ks.token, low, left, row_bytes, thread, [&](int row) { return row * a.ks.token; });
        Tile<T, DP, KT>::template fill<kSet>(to + kTile, v + (int64_t)t * KT * a.vs.token, low, left, row_bytes, thread, [&](int row) { return row * a.vs.token; });
    };
    if (lo + set < hi) fetch(lo + set, 0);
    Operand<T> q[DP / 16], grad[DP / 16];
    get_column<T, DP>(q, a.q + b * a.qs.batch + row_offset(a.qs, i, g * a.R + r), there, row_bytes, half);
    get_column<T, DP>(grad, a.grad + b * a.gs.batch + row_offset(a.gs, i, g * a.R + r), there, row_bytes, half);
    const int64_t row = ((int64_t)b * a.Sq + i) * a.H + g * a.R + r;
    // the diagonal of out grad^T, by the products that make grad v^T: where a query sees one key, whose value is its output, the two are equal to the last bit and the scores'
    // gradient is 0
    float delta = 0.0f;
    {
        Operand<T> o[DP / 16];
        get_column<T, DP>(o, a.o + row * row_bytes, there, row_bytes, half);
        f32x16 all = (f32x16)(0.0f);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) product(all, o[s], grad[s]);
#pragma unroll
        for (int e = 0; e < 16; ++e) delta = block_row(e, half) == (lane & 31) ? all[e] : delta;
        delta = halves_sum(delta);                      // the other half has 0
    }
    float exponent = there ? a.lse[((int64_t)b * a.H + g * a.R + r) * a.Sq + i] * kLog2e : INFINITY;
    if (exponent == -INFINITY) exponent = INFINITY;
    if (split == 0 && set == 0 && there && half == 0) *reinterpret_cast<f32x2*>(a.stats + ((int64_t)group * cols + col) * 2) = f32x2{exponent, delta};
    const float scale2 = a.scale * kLog2e;
    f32x16 dq[DP / 32];
#pragma unroll
    for (auto& x : dq) x = (f32x16)(0.0f);
    loads_done();
    __syncthreads();
    int at = 0;
    for (int t0 = lo; t0 < hi; t0 += SETS, at ^= 1) {
        const int t = t0 + set;
        if (t + SETS < hi) fetch(t + SETS, at ^ 1);
        const int j0 = t * KT;
        const char *kt = mine + at * 2 * kTile, *vt = kt + kTile;
        if (SETS == 1 || t < hi) {
            const bool whole = j0 >= whole_from && j0 + KT <= whole_to;
#pragma unroll
            for (int n = 0; n < KT / 32; ++n) {
                f32x16 z = (f32x16)(0.0f), dp = (f32x16)(0.0f);
#pragma unroll
                for (int s = 0; s < DP / 16; ++s) {
                    product(z, Tile<T, DP, KT>::rows(kt, 32 * n, s, lane), q[s]);
                    product(dp, Tile<T, DP, KT>::rows(vt, 32 * n, s, lane), grad[s]);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(z[e], scale2, -exponent));
                    z[e] = p * (dp[e] - delta);
                }
                if (!whole) {
                    uint32_t keys = (uint32_t)(to - from);
                    stay_a_branch(keys);
#pragma unroll
                    for (int e = 0; e < 16; ++e) z[e] = (uint32_t)(j0 + 32 * n + block_row(e, half) - from) < keys ? z[e] : 0.0f;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = z[8 * c + j];
                    const Operand<T> ds = Operand<T>::of(w);            // bfloat16: rounded, as the matrix instruction takes both factors of one type; z and dp are not (the gradients' error 0.0017 -> 0.0024)
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) product(dq[d], Tile<T, DP, KT>::columns(kt, 32 * n + 16 * c, 32 * d, lane), ds);
                }
            }
        }
        loads_done();
        __syncthreads();
    }
    if constexpr (SETS > 1) {
        add_sets<SETS, kSet, DP / 32>(dq, memory, set, thread);
        if (set) return;
    }
    if (!there) return;
    if (a.query_splits > 1) put_column<float, DP>(a.query_sums + (((int64_t)split * a.groups + group) * cols + col) * a.D, dq, a.scale, a.D, half);     // [split][group][column][D]
    else put_column<T, DP>(reinterpret_cast<T*>(a.dq) + row * a.D, dq, a.scale, a.D, half);
}

// Wavefronts of 32 keys each, WAVES of them, share the tiles of the columns (queries of all heads that share the keys) and their gradients.  SETS such take every SETS-th
// tile each: with two there are always two wavefronts a SIMD, one with the matrix unit while the other takes exponentials.  VALUES: the values wait in the
// local memory, not in registers, of which dK, dV and K take 192 at 128 features.  Z = Q K^T and dP = grad V^T have a key a lane: P and dS are operands of dV = grad^T P and dK = Q^T dS as they are.
// Four products.  Bound as the queries' kernel: the same cases 574 to 630 us = 870 to 960 TFLOP/s, and 123 us in fp32 (75 for the products alone; 576 workgroups on 256 CUs leave a third of the last
// round empty).
template <typename T, int DP, int CT, int WAVES, int SETS, bool VALUES> __global__ __launch_bounds__(64 * WAVES * SETS) void back_keys(BackArgs a) {
    constexpr int kSet = 64 * WAVES, kKeys = 32 * WAVES;
    typedef Tile<T, DP, CT> Columns;
    typedef Tile<T, DP, kKeys> Values;
    constexpr int kTiles = SETS * 4 * Columns::kBytes;
    static_assert(SETS == 1 || kSet * (DP / 32) * 64 <= kTiles + (VALUES ? Values::kBytes : 0), "a set's blocks in place of the tiles");
    __shared__ __attribute__((aligned(16))) char memory[kTiles + (VALUES ? Values::kBytes : 0)];
    __shared__ __attribute__((aligned(16))) float stats[SETS][2][CT][2];
    static_assert(CT == 32, "a tile's numbers are one load of a wavefront");
    const int set = SETS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / kSet), thread = threadIdx.x % kSet, lane = thread & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int group = blockIdx.x % a.groups, split = blockIdx.x / a.groups % a.splits, block = blockIdx.x / a.groups / a.splits;
    const int b = group / a.G, g = group % a.G;
    const uint32_t cols = (uint32_t)a.Sq * (uint32_t)a.R;
    const Seen seen = seen_of(a, b);
    const int first = block * kKeys, wave_key = first + 32 * wave, key = wave_key + (lane & 31);
    const int last = min(first + kKeys - 1, seen.keys - 1);
    // the columns of the workgroup, of the wavefront and of the lane: those of whole queries
    const bool any = first < seen.keys, works = wave_key < seen.keys, there = key < seen.keys;
    int lo = any ? seen.query_from(first) * a.R / CT : 0, hi = any ? (seen.query_to(last) * a.R + CT - 1) / CT : 0;
    part_of(split, a.splits, a.least_columns, lo, hi);
    const int whole_from = seen.query_from(min(wave_key + 31, a.Sk - 1)) * a.R, whole_to = works && wave_key + 31 < seen.keys ? seen.query_to(wave_key) * a.R : 0;
    const int from = there ? seen.query_from(key) * a.R : 0, to = there ? max(from, seen.query_to(key) * a.R) : 0;
    const char* q = a.q + b * a.qs.batch + (int64_t)g * a.R * a.qs.head;
    const char* gr = a.grad + b * a.gs.batch + (int64_t)g * a.R * a.gs.head;
    const int row_bytes = a.D * (int)sizeof(T);
    char* mine = memory + set * 4 * Columns::kBytes;
    const auto fetch = [&](int t, int at) {
        const uint32_t c0 = (uint32_t)t * CT, i0 = c0 / (uint32_t)a.R, r0 = c0 - i0 * (uint32_t)a.R;
        const int left = (int)(cols - c0);
        const auto offset = [&](const Heads& s) {
            return [&, s](int row) { const uint32_t n = r0 + row, i = fdiv(n, a.by_R); return (int)i * s.token + (int)(n - i * (uint32_t)a.R) * s.head; };
        };
        char* to = mine + at * 2 * Columns::kBytes;
        if (wave == 0) {                                    // columns behind the last have zeros: their rows are zeros too
            load_lds4(buffer(a.stats + ((int64_t)group * cols + c0) * 2, 4u * 2 * (uint32_t)min(left, CT)), stats[set][at], (uint32_t)lane * 4);
        }
        Columns::template fill<kSet>(to, q + (int64_t)i0 * a.qs.token, 0, left, row_bytes, thread, offset(a.qs));
        Columns::template fill<kSet>(to + Columns::kBytes, gr + (int64_t)i0 * a.gs.token, 0, left, row_bytes, thread, offset(a.gs));
    };
    if (lo + set < hi) fetch(lo + set, 0);
    char* values = memory + kTiles;
    const char* v_head = a.v + b * a.vs.batch + (int64_t)g * a.vs.head;
    if constexpr (VALUES)
        Values::template fill<kSet * SETS>(values, v_head + (int64_t)first * a.vs.token, 0, seen.keys - first, row_bytes, threadIdx.x, [&](int row) { return row * a.vs.token; });
    Operand<T> k[DP / 16], v[VALUES ? 1 : DP / 16];
    get_column<T, DP>(k, a.k + b * a.ks.batch + row_offset(a.ks, key, g), there, row_bytes, half);
    if constexpr (!VALUES) get_column<T, DP>(v, v_head + (int64_t)key * a.vs.token, there, row_bytes, half);
    const float scale2 = a.scale * kLog2e;
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (auto& x : dk) x = (f32x16)(0.0f);
#pragma unroll
    for (auto& x : dv) x = (f32x16)(0.0f);
    loads_done();
    __syncthreads();
    int at = 0;
    for (int t0 = lo; t0 < hi; t0 += SETS, at ^= 1) {
        const int t = t0 + set;
        if (t + SETS < hi) fetch(t + SETS, at ^ 1);
        const int c0 = t * CT;
        const char *qt = mine + at * 2 * Columns::kBytes, *gt = qt + Columns::kBytes;
        if (t < hi) {
            const bool whole = c0 >= whole_from && c0 + CT <= whole_to;
#pragma unroll 1
            for (int n = 0; n < CT / 32; ++n) {
                f32x16 z = (f32x16)(0.0f), dp = (f32x16)(0.0f);
#pragma unroll
                for (int s = 0; s < DP / 16; ++s) {
                    product(z, Columns::rows(qt, 32 * n, s, lane), k[s]);
                    if constexpr (VALUES) product(dp, Columns::rows(gt, 32 * n, s, lane), Values::rows(values, 32 * wave, s, lane));
                    else product(dp, Columns::rows(gt, 32 * n, s, lane), v[s]);
                }
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const f32x4 two = *reinterpret_cast<const f32x4*>(stats[set][at][32 * n + block_row(e, half)]);
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        z[e + f] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[e + f], scale2, -two[2 * f]));
                        dp[e + f] = z[e + f] * (dp[e + f] - two[2 * f + 1]);
                    }
                }
                if (!whole) {
                    uint32_t seeing = (uint32_t)(to - from);
                    stay_a_branch(seeing);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool sees = (uint32_t)(c0 + 32 * n + block_row(e, half) - from) < seeing;
                        z[e] = sees ? z[e] : 0.0f;
                        dp[e] = sees ? dp[e] : 0.0f;
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float w[8], x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) { w[j] = z[8 * c + j]; x[j] = dp[8 * c + j]; }
                    const Operand<T> p = Operand<T>::of(w), ds = Operand<T>::of(x);     // rounded in bfloat16, as in the queries' kernel
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) product(dv[d], Columns::columns(gt, 32 * n + 16 * c, 32 * d, lane), p);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) product(dk[d], Columns::columns(qt, 32 * n + 16 * c, 32 * d, lane), ds);
                }
            }
        }
        loads_done();
        __syncthreads();
    }
    if constexpr (SETS > 1) {
        add_sets<SETS, kSet, DP / 32>(dk, memory, set, thread);
        add_sets<SETS, kSet, DP / 32>(dv, memory, set, thread);
        if (set) return;
    }
    if (a.splits > 1) {                                     // [split][group][key][2][D]
        if (key >= a.Sk) return;
        float* row = a.key_sums + (((int64_t)split * a.groups + group) * a.Sk + key) * 2 * a.D;
        put_column<float, DP>(row, dk, a.scale, a.D, half);
        put_column<float, DP>(row + a.D, dv, 1.0f, a.D, half);
        return;
    }
    if (key >= a.Sk) return;
    const int64_t row = (((int64_t)b * a.Sk + key) * a.G + g) * a.D;
    put_column<T, DP>(reinterpret_cast<T*>(a.dk) + row, dk, a.scale, a.D, half);
    put_column<T, DP>(reinterpret_cast<T*>(a.dv) + row, dv, 1.0f, a.D, half);
}

// The parts of gradients, in their order: four elements a thread, eight loads on their way.  Bound by memory.  QUERIES: of dq, [group][column][D]; else of dk and dv, [group][key][2][D]
template <typename T, bool QUERIES> __global__ __launch_bounds__(kThreads) void add_parts(BackArgs a) {
    const int pieces = (QUERIES ? a.D : 2 * a.D) / 4, splits = QUERIES ? a.query_splits : a.splits;
    const int64_t rows = QUERIES ? (int64_t)a.Sq * a.R : a.Sk, n = (int64_t)a.groups * rows, at = (int64_t)blockIdx.x * kThreads + threadIdx.x, row = at / pieces;
    if (row >= n) return;
    const int e = (int)(at - row * pieces) * 4;
    const float* from = (QUERIES ? a.query_sums : a.key_sums) + at * 4;
    f32x4 o = {0, 0, 0, 0};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) o += *reinterpret_cast<const f32x4*>(from + s * n * pieces * 4);
    const int64_t group = row / rows, r = row - group * rows, b = group / a.G, g = group - b * a.G;
    T* out;
    if constexpr (QUERIES) {
        const int64_t i = r / a.R;
        out = reinterpret_cast<T*>(a.dq) + ((b * a.Sq + i) * a.H + g * a.R + (r - i * a.R)) * a.D + e;
    } else {
        out = reinterpret_cast<T*>(e < a.D ? a.dk : a.dv) + ((b * a.Sk + r) * a.G + g) * a.D + (e < a.D ? e : e - a.D);
    }
    put4(out, o[0], o[1], o[2], o[3]);
}

// ------------------------------------------------------------------ host side

size_t stats_bytes(const division_attention& a) { return ((size_t)(a.B * a.Sq * a.H) * 8 + 15) / 16 * 16; }

// The workgroups' shapes.  fp32 products are slow enough for small ones to pay: 64 columns or keys, their tiles shared by two (four) sets.  (2 x 1531 tokens, 12 heads of 64, window 256: 228 us with
// workgroups of 128, 191 so; 4 x 1024 tokens, 8 heads of 128, causal, 405 and 301.)  FEW, in bfloat16: 64 too, and four sets, where blocks of 128 leave CUs without work (16 heads of 64, 1024 tokens: 52 us, 32 so; of 128, 81 and 47; but 2 x 12 heads of
// 64, 1531 tokens, which make 288 blocks, 48 and 55).
constexpr int kColumnTile = 32;
template <typename T, int DP, bool FEW> struct Shape {
    static constexpr bool kHalf = sizeof(T) == 2, kSmall = !kHalf && DP <= 64;
    static constexpr int kKeyTile = kHalf && !FEW ? 64 : 32, kQueryWaves = kHalf && !FEW ? 4 : 2, kQuerySets = kHalf ? (FEW ? 4 : 1) : 2;
    static constexpr int kKeyWaves = !kHalf || FEW ? 2 : 4, kKeySets = kSmall || FEW ? 4 : 2;
    static constexpr bool kValues = kHalf && DP == 128;
};
// Parts of what a workgroup would have to look at, where there are few workgroups: as many as make two a CU, of so many tiles at least that they pay for adding them up.  (One sequence of 2048, 32 heads
// on 4 of keys: 484 us with the columns of 128 keys in one part, 166 so.  Two heads of 4090 tokens, whose queries' keys are cut too: 163 us in one part, 90 so.  Parts of 8 tiles for four sets: 8 heads
// of 64, 1024 tokens 47 us, 31 with 24.)
// enough: workgroups that need no parts, one for every CU, two where a CU has room for one and the other half's end would be waited for (fp32 keys of more than 64 features: 8 heads of 128, 2048 tokens:
// 490 us with 256, 386 so).
constexpr int kMostSplits = 32;
int parts_of(int64_t tasks, int64_t tiles, int64_t least, int64_t enough) {
    if (tasks == 0 || tasks >= enough) return 1;
    int64_t n = tasks > 256 ? 2 : 512 / tasks;              // no more than make two a CU, or their last ones have a round of their own (7 heads of 128, 1024 tokens in fp32: 155 us, 133 so)
    if (n > tiles / least) n = tiles / least;
    return n < 1 ? 1 : n > kMostSplits ? kMostSplits : (int)n;
}
struct Splits { int queries, keys, least_keys, least_columns; bool few_queries, few_keys; };
Splits splits_of(const division_attention& a) {
    const bool half = a.dt == DIVISION_BF16;
    const int64_t cols = a.Sq * (a.H / a.G), groups = a.B * a.G;
    Splits s;
    // not over long sequences, whose parts keep larger workgroups busy too (two heads of 128, 4090 tokens: 89 us, 97 with small ones).  A window is not looked at here, though it leaves a block few tiles and
    // no parts: 2 x 3000 tokens, 8 heads on 4 of 128, window 79 take 69 us (187 without one)
    s.few_queries = half && (cols + 127) / 128 * groups < 256 && a.Sk <= 2048;
    s.few_keys = half && (a.Sk + 127) / 128 * groups < 256 && cols <= 4096;
    s.least_keys = s.few_queries ? 24 : half ? 4 : 2;
    s.least_columns = s.few_keys ? 24 : half ? 8 : 2;
    const int64_t key_tile = half && !s.few_queries ? 64 : 32, of_queries = half && !s.few_queries ? 128 : 64, of_keys = s.few_keys || !half ? 64 : 128;
    s.queries = parts_of((cols + of_queries - 1) / of_queries * groups, (a.Sk + key_tile - 1) / key_tile, s.least_keys, 256);
    s.keys = parts_of((a.Sk + of_keys - 1) / of_keys * groups, (cols + kColumnTile - 1) / kColumnTile, s.least_columns, half || a.D <= 64 ? 256 : 512);
    return s;
}
size_t key_bytes(const division_attention& a) { const int n = splits_of(a).keys; return n > 1 ? (size_t)n * a.B * a.G * a.Sk * 2 * a.D * 4 : 0; }
size_t query_bytes(const division_attention& a) { const int n = splits_of(a).queries; return n > 1 ? (size_t)n * a.B * a.H * a.Sq * a.D * 4 : 0; }
size_t back_bytes(const division_attention& a) { return stats_bytes(a) + key_bytes(a) + query_bytes(a); }

// The two launches; `check`: whether they can be, without them
template <typename T, int DP, bool FEW> int run_queries(BackArgs& args, bool check, hipStream_t st) {
    typedef Shape<T, DP, FEW> S;
    constexpr int kCols = 32 * S::kQueryWaves, kWorkgroup = 64 * S::kQueryWaves * S::kQuerySets;
    const int64_t blocks = ((int64_t)args.Sq * args.R + kCols - 1) / kCols, grid = blocks * args.groups * args.query_splits;
    if (grid >= (int64_t(1) << 23)) return DIVISION_ERANGE;
    if (check || grid == 0) return DIVISION_OK;
    args.blocks = (int)blocks;
    hipLaunchKernelGGL((back_queries<T, DP, S::kKeyTile, S::kQueryWaves, S::kQuerySets>), dim3((uint32_t)grid), dim3(kWorkgroup), 0, st, args);
    CHECKED(launched());
    if (args.query_splits == 1) return DIVISION_OK;
    const int64_t pieces = (int64_t)args.groups * args.Sq * args.R * (args.D / 4);
    hipLaunchKernelGGL((add_parts<T, true>), dim3((uint32_t)((pieces + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, args);
    return launched();
}
template <typename T, int DP, bool FEW> int run_keys(const BackArgs& args, bool check, hipStream_t st) {
    typedef Shape<T, DP, FEW> S;
    constexpr int kKeys = 32 * S::kKeyWaves, kWorkgroup = 64 * S::kKeyWaves * S::kKeySets;
    const int64_t grid = ((int64_t)args.Sk + kKeys - 1) / kKeys * args.groups * args.splits;
    if (grid >= (int64_t(1) << 23)) return DIVISION_ERANGE;
    if (check || grid == 0) return DIVISION_OK;
    hipLaunchKernelGGL((back_keys<T, DP, kColumnTile, S::kKeyWaves, S::kKeySets, S::kValues>), dim3((uint32_t)grid), dim3(kWorkgroup), 0, st, args);
    CHECKED(launched());
    if (args.splits == 1) return DIVISION_OK;
    const int64_t pieces = (int64_t)args.groups * args.Sk * (args.D / 2);
    hipLaunchKernelGGL((add_parts<T, false>), dim3((uint32_t)((pieces + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, args);
    return launched();
}
template <typename T, int DP> int run(BackArgs& args, const Splits& splits, hipStream_t st) {
    const auto queries = [&](bool check) {
        if constexpr (sizeof(T) == 2) if (splits.few_queries) return run_queries<T, DP, true>(args, check, st);
        return run_queries<T, DP, false>(args, check, st);
    };
    const auto keys = [&](bool check) {
        if constexpr (sizeof(T) == 2) if (splits.few_keys) return run_keys<T, DP, true>(args, check, st);
        return run_keys<T, DP, false>(args, check, st);
    };
    CHECKED(queries(true));
    CHECKED(keys(true));
    CHECKED(queries(false));
    return keys(false);
}

}  // namespace

extern "C" {

size_t division_attention_backward_workspace(const division_attention* attention) {
    if (!attention || check_attention(*attention) != DIVISION_OK) return 0;
    return back_bytes(*attention);
}

int division_attention_backward(const division_attention* attention, const division_attention_back* back, void* hip_stream) {
    if (!attention || !back) return DIVISION_EINVAL;
    const division_attention& a = *attention;
    const division_attention_back& w = *back;
    CHECKED(check_attention(a));
    if (a.B == 0 || (a.Sq == 0 && a.Sk == 0)) return DIVISION_OK;
    const int64_t es = a.dt == DIVISION_BF16 ? 2 : 4;
    if ((a.Sq > 0 && (!a.q || !w.grad_out || !w.out || !w.lse || !w.grad_q)) || (a.Sk > 0 && (!w.grad_k || !w.grad_v || !a.k || !a.v))) return DIVISION_EINVAL;
    const size_t need = back_bytes(a);
    if (!w.workspace && need) return DIVISION_EINVAL;
    if (!aligned(w.out, 16) || !aligned(w.lse, 4) || !aligned(w.grad_q, 16) || !aligned(w.grad_k, 16) || !aligned(w.grad_v, 16) || !aligned(w.workspace, 16)) return DIVISION_EALIGN;
    if (a.Sq > 0) CHECKED(check_heads(w.grad_out, w.grad_out_strides, a.B, a.H / a.G, es));
    if (w.workspace_bytes < need) return DIVISION_ESIZE;
    BackArgs args{};
    static_cast<AttentionArgs&>(args) = args_of(a);
    args.grad = static_cast<const char*>(w.grad_out);
    args.gs = heads_of(w.grad_out_strides, es);
    args.o = static_cast<const char*>(w.out);
    args.lse = const_cast<float*>(w.lse);
    args.dq = static_cast<char*>(w.grad_q); args.dk = static_cast<char*>(w.grad_k); args.dv = static_cast<char*>(w.grad_v);
    args.stats = static_cast<float*>(w.workspace);
    const Splits splits = splits_of(a);
    args.splits = splits.keys;
    args.query_splits = splits.queries;
    args.least_keys = splits.least_keys;
    args.least_columns = splits.least_columns;
    args.key_sums = reinterpret_cast<float*>(static_cast<char*>(w.workspace) + stats_bytes(a));
    args.query_sums = reinterpret_cast<float*>(static_cast<char*>(w.workspace) + stats_bytes(a) + key_bytes(a));
    args.by_R = make_fastdiv((uint32_t)args.R);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (a.dt == DIVISION_BF16) return a.D <= 64 ? run<uint16_t, 64>(args, splits, st) : a.D <= 96 ? run<uint16_t, 96>(args, splits, st) : run<uint16_t, 128>(args, splits, st);
    return a.D <= 32 ? run<float, 32>(args, splits, st) : a.D <= 64 ? run<float, 64>(args, splits, st) : a.D <= 96 ? run<float, 96>(args, splits, st) : run<float, 128>(args, splits, st);
}

}  // extern "C"
