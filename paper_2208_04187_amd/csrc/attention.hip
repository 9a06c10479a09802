// Attention of a token model for AMD MI355X (gfx950).
//
//   z = scale q k^T over the keys that a query sees;   out = softmax(z) v;   lse = ln(sum of exp(z))
//
// One pass over the keys with the running maximum and sum of each query's exponentials; scores and probabilities stay in registers.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"
#include "tiles.h"
#include "attention_args.h"

// What a wavefront holds of 32 columns: their running maximum (of the raw scores), sum and weighted values, [DP elements][columns] in blocks of 32 x 32
template <typename T, int DP> struct Columns {
    f32x16 o[DP / 32];
    float most, total;                                      // both halves of a column have the maximum; each its own rows' part of the sum
    Operand<T> q[DP / 16];

    __device__ __forceinline__ void begin(const AttentionArgs& a, const char* q_head, uint32_t col, uint32_t cols, int half) {
#pragma unroll
        for (auto& b : o) b = (f32x16)(0.0f);
        most = -INFINITY;
        total = 0.0f;
        const uint32_t i = col / (uint32_t)a.R, r = col % (uint32_t)a.R;
        const char* row = q_head + row_offset(a.qs, i, (int)r);
        const int row_bytes = a.D * (int)sizeof(T);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            const int at = (16 * s + 8 * half) * (int)sizeof(T);
            q[s] = col < cols && at < row_bytes ? Operand<T>::at(row + at) : Operand<T>::zero();
        }
    }

    // KT keys of the tiles, the first of them key `first`; from .. to - 1 are the keys that this lane's column sees, all of these where `whole`
    template <typename Keys, int KT> __device__ __forceinline__ void add(const char* kt, const char* vt, int first, int from, int to, bool whole, float scale2, int lane) {
        const int half = lane >> 5;
        f32x16 z[KT / 32];
#pragma unroll
        for (auto& b : z) b = (f32x16)(0.0f);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
#pragma unroll
            for (int b = 0; b < KT / 32; ++b) product(z[b], Keys::rows(kt, 32 * b, s, lane), q[s]);
        if (!whole) {
            uint32_t n = (uint32_t)(to - from);
            stay_a_branch(n);
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[b][i] = (uint32_t)(first + 32 * b + block_row(i, half) - from) < n ? z[b][i] : -INFINITY;
        }
        float m = z[0][0];
#pragma unroll
        for (int b = 0; b < KT / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, z[b][i]);
        m = halves_max(m);
        // The maximum that exponents are taken against need not be the largest yet: sums and products stay exact to their last bits while they grow by at most 2^8, so that most tiles leave
        // the weighted values alone
        if (__any((m - most) * scale2 > 8.0f || most == -INFINITY)) {
            stay_a_branch(m);
            m = fmaxf(m, most);
            const float shrink = most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((most - m) * scale2);
            total *= shrink;
#pragma unroll
            for (auto& b : o)
#pragma unroll
                for (int i = 0; i < 16; ++i) b[i] *= shrink;
            most = m;
        }
        const float by = most == -INFINITY ? 0.0f : most * scale2;
#pragma unroll
        for (int b = 0; b < KT / 32; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][i], scale2, -by));
#pragma unroll
            for (int i = 0; i < 16; ++i) total += z[b][i];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = z[b][8 * c + j];
                // bfloat16: rounded, as the matrix instruction takes both factors of one type, by half a step of 2^-8 each; `total` has them unrounded.  (Error of the output, as a norm, against 64 bits: 0.0016 for
                // the output's own rounding, 0.0021 with this one; a second product of what the rounding left out would keep it, for half as many products again.)
                const Operand<T> p = Operand<T>::of(w);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) product(o[d], Keys::columns(vt, 32 * b + 16 * c, 32 * d, lane), p);
            }
        }
    }
};

// The workgroup's part of the tiles lo .. hi - 1 that its columns see: equal parts of these, not of all keys, or the long sequences of a batch would leave most of their parts' workgroups without work
// (32 tokens over caches of up to 8192 keys: 78 us, 71 so)
__device__ __forceinline__ void part_of(const AttentionArgs& a, int split, int& lo, int& hi) {
    const int each = max((hi - lo + a.splits - 1) / a.splits, a.tiles), begin = lo + split * each;
    hi = min(begin + each, hi);
    lo = begin;
}

constexpr int kThreads = 256;

// Four wavefronts of 32 columns each share the tiles of the keys, two tiles of 64 keys in the local memory, the second on its way while the first is looked at.  S = K Q^T, so that a lane has one
// query's scores and its maximum and sum are one exchange between two lanes, and P's registers are the operand of O = V^T P as they are.  The heads that share a key head are columns of one workgroup: its
// keys are read once for all of them.
// Bound by the matrix unit's power: 2 x 4096 tokens, 32 heads on 8 of 128 in bfloat16, causal, 281 us = 990 TFLOP/s of the visible pairs (a large product reaches 1250; the same instructions on
// zeros take 220 us).  Neither operands read a use ahead, nor three tiles, nor three wavefronts a SIMD changed that (275 to 288), and 64 columns a wavefront took 361.
template <typename T, int DP, int KT> __global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void attend(AttentionArgs a) {
    constexpr int kTile = Tile<T, DP, KT>::kBytes;
    __shared__ __attribute__((aligned(16))) char tiles[2][2][kTile];
    const int thread = threadIdx.x, lane = thread & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int group = blockIdx.x % a.groups, split = blockIdx.x / a.groups % a.splits, block = a.blocks - 1 - blockIdx.x / a.groups / a.splits;
    const int b = group / a.G, g = group % a.G;
    const uint32_t cols = (uint32_t)a.Sq * (uint32_t)a.R, first_col = (uint32_t)block * 128u;
    const uint32_t wave_col = first_col + 32 * wave, col = wave_col + (lane & 31);
    const Seen seen = seen_of(a, b);
    const int first_key = seen.from(0);                     // what stands before every query's keys is not looked at either
    // the keys of the workgroup, of the wavefront and of the lane
    const uint32_t last_col = min(first_col + 127u, cols - 1), wave_last = min(wave_col + 31u, cols - 1);
    int lo = seen.from((int)(first_col / (uint32_t)a.R)) / KT, hi = (seen.to((int)(last_col / (uint32_t)a.R)) + KT - 1) / KT;
    part_of(a, split, lo, hi);
    const int qa = wave_col < cols ? (int)(wave_col / (uint32_t)a.R) : 0, qb = wave_col < cols ? (int)(wave_last / (uint32_t)a.R) : 0;
    const int whole_from = seen.from(qb), whole_to = seen.to(qa);
    const int i = (int)(min(col, cols - 1) / (uint32_t)a.R);
    const int from = seen.from(i), to = col < cols ? max(from, seen.to(i)) : from;
    const char* k = a.k + b * a.ks.batch + (int64_t)g * a.ks.head;
    const char* v = a.v + b * a.vs.batch + (int64_t)g * a.vs.head;
    const int row_bytes = a.D * (int)sizeof(T);
    const auto fetch = [&](int t) {
        const int low = first_key - t * KT, left = seen.keys - t * KT;
        Tile<T, DP, KT>::template fill<kThreads>(tiles[t & 1][0], k + (int64_t)t * KT * a.ks.token, low, left, row_bytes, thread, [&](int row) { return row * a.ks.token; });
        Tile<T, DP, KT>::template fill<kThreads>(tiles[t & 1][1], v + (int64_t)t * KT * a.vs.token, low, left, row_bytes, thread, [&](int row) { return row * a.vs.token; });
    };
    if (lo < hi) fetch(lo);
    Columns<T, DP> c;
    c.begin(a, a.q + b * a.qs.batch + (int64_t)g * a.R * a.qs.head, col, cols, half);
    const float scale2 = a.scale * kLog2e;
    loads_done();
    __syncthreads();
    for (int t = lo; t < hi; ++t) {
        if (t + 1 < hi) fetch(t + 1);
        const int j = t * KT;
        c.template add<Tile<T, DP, KT>, KT>(tiles[t & 1][0], tiles[t & 1][1], j, from, to, j >= whole_from && j + KT <= whole_to, scale2, lane);
        loads_done();
        __syncthreads();
    }
    if (col >= cols) return;
    const float total = halves_sum(c.total);
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
    const float lse = total == 0.0f ? -INFINITY : __builtin_fmaf(c.most, a.scale, logf(total));
    const int r = (int)(col % (uint32_t)a.R);
    if (a.parts) {
        const int64_t at = ((int64_t)split * a.groups + group) * cols + col;
        if (half == 0) a.parts[at] = lse;
        float* row = a.values + at * a.D;
#pragma unroll
        for (int d = 0; d < DP; d += 8) {
            if (d >= a.D) continue;
            const f32x16& o = c.o[d / 32];
            const int n = d % 32 / 2;
            *reinterpret_cast<f32x4*>(row + d + 4 * half) = f32x4{o[n] * inverse, o[n + 1] * inverse, o[n + 2] * inverse, o[n + 3] * inverse};
        }
        return;
    }
    if (half == 0) a.lse[((int64_t)b * a.H + g * a.R + r) * a.Sq + i] = lse;
    T* row = reinterpret_cast<T*>(a.out) + (((int64_t)b * a.Sq + i) * a.H + g * a.R + r) * a.D;
#pragma unroll
    for (int d = 0; d < DP; d += 8) {
        if (d >= a.D) continue;
        const f32x16& o = c.o[d / 32];
        const int n = d % 32 / 2;
        put4(row + d + 4 * half, o[n] * inverse, o[n + 1] * inverse, o[n + 2] * inverse, o[n + 3] * inverse);
    }
}

// Few columns: WK wavefronts have the same 32 columns and every WK-th tile of the keys each, in a tile of their own, and are joined at the end.  PAST: the keys are looked at by this workgroup
// alone.  Bound by memory then: 32 tokens of 32 heads on 4 of 128 over caches of up to 8192 keys in bfloat16, 56 us = 4.7 TB/s.  While a wavefront computes, seven
// others of the CU wait for their tiles; two tiles a wavefront, the second on its way, leave room for half as many (the same call: 69 us so, 64 with one tile).  In fp32 of more than 64 features a CU has room
// for one workgroup of four wavefronts or two of two, a SIMD for one wavefront, and each tile is waited for in full: the same caches in fp32 188 us = 2.9 TB/s; 3 x 777 tokens of 6 heads on 2 of 72, which see up
// to 480 and 184 keys and none, 26.6 us, where the longest wavefront has four tiles of 2.6 us of products: 9.1 if no query sees a key (438 workgroups' starts and ends, one a CU), 17.9 if 128 keys of the first
// sequence are seen (a tile a wavefront), 21.9 if its 480 are.
template <typename T, int DP, int KT, int WK, bool PAST> __global__ __launch_bounds__(64 * WK) void attend_few(AttentionArgs a) {
    typedef RowTile<T, DP, KT> Keys;
    constexpr int kTile = Keys::kBytes, kTurns = DP == 96 ? 8 : DP / 4;
    static_assert(32 * DP * 4 <= 2 * kTile, "a wavefront's values in place of its tiles");
    __shared__ __attribute__((aligned(16))) char tiles[WK][2][kTile];
    __shared__ float most[WK][32], totals[WK][32];
    const int thread = threadIdx.x, lane = thread & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int group = blockIdx.x % a.groups, split = blockIdx.x / a.groups % a.splits, block = a.blocks - 1 - blockIdx.x / a.groups / a.splits;
    const int b = group / a.G, g = group % a.G;
    const uint32_t cols = (uint32_t)a.Sq * (uint32_t)a.R, first_col = (uint32_t)block * 32u, col = first_col + (lane & 31);
    const Seen seen = seen_of(a, b);
    const int first_key = seen.from(0);                     // what stands before every query's keys is not looked at either
    const int qa = (int)(first_col / (uint32_t)a.R), qb = (int)(min(first_col + 31u, cols - 1) / (uint32_t)a.R);
    const int whole_from = seen.from(qb), whole_to = seen.to(qa);
    int lo = seen.from(qa) / KT, hi = (seen.to(qb) + KT - 1) / KT;
    part_of(a, split, lo, hi);
    const int i = (int)(min(col, cols - 1) / (uint32_t)a.R);
    const int from = seen.from(i), to = col < cols ? max(from, seen.to(i)) : from;
    const char* k = a.k + b * a.ks.batch + (int64_t)g * a.ks.head;
    const char* v = a.v + b * a.vs.batch + (int64_t)g * a.vs.head;
    const int row_bytes = a.D * (int)sizeof(T);
    const auto fetch = [&](int t) {
        const int low = first_key - t * KT, left = seen.keys - t * KT;
        Keys::template fill<64, PAST>(tiles[wave][0], k + (int64_t)t * KT * a.ks.token, low, left, row_bytes, lane, [&](int row) { return row * a.ks.token; });
        Keys::template fill<64, PAST>(tiles[wave][1], v + (int64_t)t * KT * a.vs.token, low, left, row_bytes, lane, [&](int row) { return row * a.vs.token; });
    };
    if (lo + wave < hi) fetch(lo + wave);
    Columns<T, DP> c;
    c.begin(a, a.q + b * a.qs.batch + (int64_t)g * a.R * a.qs.head, col, cols, half);
    const float scale2 = a.scale * kLog2e;
    for (int t = lo + wave; t < hi; t += WK) {
        loads_done();
        const int j = t * KT;
        c.template add<Keys, KT>(tiles[wave][0], tiles[wave][1], j, from, to, j >= whole_from && j + KT <= whole_to, scale2, lane);
        if (t + WK < hi) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the tile has been read
            fetch(t + WK);
        }
    }
    const float total = halves_sum(c.total);
    if (half == 0) { most[wave][lane] = c.most; totals[wave][lane] = total; }
    // [column][DP], pieces of four exchanged with the column's number: 32 columns at one row do not share banks
    const auto place = [](int col, int d) { return col * DP + (d / 4 ^ col % kTurns) * 4; };
    float* mine = reinterpret_cast<float*>(tiles[wave]);
#pragma unroll
    for (int d = 0; d < DP; d += 8) {
        const f32x16& o = c.o[d / 32];
        const int n = d % 32 / 2;
        *reinterpret_cast<f32x4*>(mine + place(lane & 31, d + 4 * half)) = f32x4{o[n], o[n + 1], o[n + 2], o[n + 3]};
    }
    __syncthreads();
    for (int e = thread; e < 32 * (DP / 4); e += 64 * WK) {
        const int c1 = e / (DP / 4), d = e % (DP / 4) * 4;
        const uint32_t at_col = first_col + c1;
        if (at_col >= cols || d >= a.D) continue;
        float m = most[0][c1], sum = 0.0f;
#pragma unroll
        for (int w = 1; w < WK; ++w) m = fmaxf(m, most[w][c1]);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            const float by = most[w][c1] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((most[w][c1] - m) * scale2);
            sum += by * totals[w][c1];
            o += by * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(tiles[w]) + place(c1, d));
        }
        o *= sum == 0.0f ? 0.0f : 1.0f / sum;
        const float lse = sum == 0.0f ? -INFINITY : __builtin_fmaf(m, a.scale, logf(sum));
        if (a.parts) {
            const int64_t at = ((int64_t)split * a.groups + group) * cols + at_col;
            if (d == 0) a.parts[at] = lse;
            *reinterpret_cast<f32x4*>(a.values + at * a.D + d) = o;
        } else {
            const int i1 = (int)(at_col / (uint32_t)a.R), h = g * a.R + (int)(at_col % (uint32_t)a.R);
            if (d == 0) a.lse[((int64_t)b * a.H + h) * a.Sq + i1] = lse;
            put4(reinterpret_cast<T*>(a.out) + (((int64_t)b * a.Sq + i1) * a.H + h) * a.D + d, o[0], o[1], o[2], o[3]);
        }
    }
}

// The parts of the keys of a column: out = sum of exp(lse_part - lse) out_part.  Bound by one trip to memory and the launch: 32 parts of 32 columns 3.4 us, 4 of 1024 4.7.  32 lanes have a column's elements and eight of its parts, whose loads all leave before the first wait (one after the
// other, 32 parts of 32 columns took 12 us); GROUPS such groups, joined through the local memory, where there are more.
constexpr int kMostSplits = 64, kParts = 8;
template <typename T, int GROUPS> __global__ __launch_bounds__(kThreads) void join_parts(AttentionArgs a) {
    const uint32_t cols = (uint32_t)a.Sq * (uint32_t)a.R, lane = threadIdx.x & 31, own = threadIdx.x / 32 % GROUPS;
    const uint32_t n = (uint32_t)a.groups * cols, at = blockIdx.x * (kThreads / 32 / GROUPS) + threadIdx.x / 32 / GROUPS;
    if (GROUPS == 1 && at >= n) return;
    const int d = (int)lane * 4;
    const float* from = a.values + (int64_t)at * a.D + (d < a.D ? d : 0);
    float lses[kParts], most = -INFINITY;
    f32x4 parts[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {                      // behind the last part that again, which counts for nothing: no load waits for a branch
        const int s = (int)own + k * GROUPS;
        const int64_t row = (int64_t)(s < a.splits ? s : a.splits - 1) * n;
        const float lse = a.parts[row + at];
        lses[k] = s < a.splits ? lse : -INFINITY;
        parts[k] = *reinterpret_cast<const f32x4*>(from + row * a.D);
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) most = fmaxf(most, lses[k]);
    f32x4 o = {0, 0, 0, 0};
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kParts; ++k) {                      // a part that saw no key has zeros
        const float by = lses[k] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((lses[k] - most) * kLog2e);
        sum += by;
        o += by * parts[k];
    }
    if constexpr (GROUPS > 1) {
        __shared__ float mosts[GROUPS], sums[GROUPS];
        __shared__ f32x4 values[GROUPS][32];
        values[own][lane] = o;
        if (lane == 0) { mosts[own] = most; sums[own] = sum; }
        __syncthreads();
        if (own) return;
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) most = fmaxf(most, mosts[k]);
        o = f32x4{0, 0, 0, 0};
        sum = 0.0f;
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            const float by = mosts[k] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mosts[k] - most) * kLog2e);
            sum += by * sums[k];
            o += by * values[k][lane];
        }
    }
    o *= sum == 0.0f ? 0.0f : 1.0f / sum;
    const uint32_t group = at / cols, col = at - group * cols, i = col / (uint32_t)a.R;
    const int b = (int)group / a.G, h = (int)group % a.G * a.R + (int)(col - i * (uint32_t)a.R);
    if (d == 0) a.lse[((int64_t)b * a.H + h) * a.Sq + i] = sum == 0.0f ? -INFINITY : most + logf(sum);
    if (d < a.D) put4(reinterpret_cast<T*>(a.out) + (((int64_t)b * a.Sq + i) * a.H + h) * a.D + d, o[0], o[1], o[2], o[3]);
}

// ------------------------------------------------------------------ host side

// How the work is cut: columns into blocks, of 128 for attend or of 32 for attend_few, and the keys into parts where that leaves CUs without work.
//   one block of 32 (few queries): attend_few, 1024 workgroups, four a CU, of eight tiles at least (32 tokens over caches of up to 8192 keys: 63 us with 512, 60 so); 256 of four at least where there
//   are not so many keys (one token of 32 heads on 8 over 4097: 11.3 us with eight, 10.4 with four);
//   blocks of 128 that leave CUs or matrix units without work: attend_few too, whose wavefronts share the keys of 32 columns without a second kernel.  bfloat16, 16 heads of 64, 1024 tokens: 23.4 us
//   from attend, 11.3 so, 16 heads of 128 26.8 and 17.3, 32 heads of 64, 512 tokens 17.3 and 8.3; but, since a tile is read for fewer columns, 64 tokens of 32 heads on 8 over 16000 keys 24 and 34, 32
//   heads of 128, 1000 tokens 24.8 and 27.5, hence the limits.  fp32, 8 heads of 64, 4 x 1024 tokens: 77 and 57, 777 tokens of 6 heads of 72 35 and 28, but 16 x 256 tokens of 16 heads of 64 36 and 47.
//   256 workgroups at least, 512 where fp32 sequences are long (4 heads of 128, 2048 tokens: 84 and 65 us; 8 heads, 1024 tokens 47 and 59);
//   else attend, in bfloat16 over long sequences with 512 workgroups of four tiles at least.
struct Cut { bool few; int64_t blocks; int splits, tiles; };
Cut cut_of(const division_attention& a) {
    Cut c;
    const int64_t R = a.H / a.G, cols = a.Sq * R, half = a.dt == DIVISION_BF16;
    const int64_t wide = (cols + 127) / 128 * a.B * a.G;
    c.few = cols <= 32 || (half ? a.Sk <= 2048 && (wide <= 128 || (wide < 256 && a.Sk >= 512 && (a.D <= 64 || a.D > 96))) : wide < (a.Sk < 1024 ? 256 : a.D <= 64 ? 512 : 320));
    c.blocks = (cols + (c.few ? 31 : 127)) / (c.few ? 32 : 128);
    const int64_t tile = c.few ? 32 : 64, tiles = (a.Sk + tile - 1) / tile, tasks = c.blocks * a.B * a.G;
    const auto parts = [&](int64_t wanted, int64_t least) {
        c.tiles = (int)least;
        const int64_t n = (wanted + tasks - 1) / tasks, room = tiles / least;
        c.splits = (int)(n > room ? room : n);
        if (c.splits > kMostSplits) c.splits = kMostSplits;
        if (c.splits < 1) c.splits = 1;
    };
    if (c.few) {
        parts(cols <= 32 ? 1024 : half || a.Sk < 2048 ? 256 : 512, half ? 8 : 4);
        if (cols <= 32 && tasks * c.splits < 256) parts(256, half ? 4 : 2);
    } else if (tasks < 256) {
        parts(512, 4);
    } else {
        parts(tasks, 1);
    }
    return c;
}
size_t lse_bytes(const division_attention& a, const Cut& c) { return ((size_t)c.splits * a.B * a.Sq * a.H * 4 + 15) / 16 * 16; }
size_t parts_bytes(const division_attention& a, const Cut& c) { return c.splits > 1 ? lse_bytes(a, c) + (size_t)c.splits * a.B * a.Sq * a.H * a.D * 4 : 0; }

template <typename T, int DP> int run(const AttentionArgs& args, const Cut& c, int64_t grid, hipStream_t st) {
    constexpr bool kFew = sizeof(T) == 4 || DP != 96;                                // 96 bfloat16 are no rows of eight pieces: few columns of such heads take 128
    if constexpr (kFew) {
        // keys that one block of columns looks at are looked at once.  In fp32 two wavefronts, so that two workgroups fit a CU's local memory, unless there are no two (16 tokens over 2000 keys, 8 heads of
        // 128: 80 us with four, 69 so; one token of 32 heads on 8 over 4000: 19 us with two, 14 so)
        void (*few)(AttentionArgs) = c.blocks > 1 ? attend_few<T, DP, 32, 4, false> : attend_few<T, DP, 32, 4, true>;
        int waves = 4;
        if constexpr (sizeof(T) == 4) {
            if (c.blocks == 1 && grid > 256) { few = attend_few<T, DP, 32, 2, true>; waves = 2; }
        }
        if (c.few) hipLaunchKernelGGL(few, dim3((uint32_t)grid), dim3(64 * waves), 0, st, args);
    }
    if (!c.few) hipLaunchKernelGGL((attend<T, DP, 64>), dim3((uint32_t)grid), dim3(kThreads), 0, st, args);
    CHECKED(launched());
    if (c.splits == 1) return DIVISION_OK;
    const int64_t rows = (int64_t)args.groups * args.Sq * args.R;
    if (c.splits <= kParts) hipLaunchKernelGGL((join_parts<T, 1>), dim3((uint32_t)((rows + 7) / 8)), dim3(kThreads), 0, st, args);
    else hipLaunchKernelGGL((join_parts<T, kMostSplits / kParts>), dim3((uint32_t)rows), dim3(kThreads), 0, st, args);
    return launched();
}

}  // namespace

extern "C" {

size_t division_attention_workspace(const division_attention* attention) {
    if (!attention || check_attention(*attention) != DIVISION_OK || attention->B == 0 || attention->Sq == 0) return 0;
    return parts_bytes(*attention, cut_of(*attention));
}

int division_attend(const division_attention* attention, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!attention) return DIVISION_EINVAL;
    const division_attention& a = *attention;
    CHECKED(check_attention(a));
    if (a.B == 0 || a.Sq == 0) return DIVISION_OK;
    if (!a.q || (a.Sk > 0 && (!a.k || !a.v)) || !out || !lse) return DIVISION_EINVAL;
    if (!aligned(out, 16) || !aligned(lse, 4)) return DIVISION_EALIGN;
    const Cut c = cut_of(a);
    const size_t need = parts_bytes(a, c);
    if (need && !workspace) return DIVISION_EINVAL;
    if (need && !aligned(workspace, 16)) return DIVISION_EALIGN;
    if (workspace_bytes < need) return DIVISION_ESIZE;
    AttentionArgs args = args_of(a);
    args.out = static_cast<char*>(out);
    args.lse = lse;
    args.parts = need ? static_cast<float*>(workspace) : nullptr;
    args.values = need ? reinterpret_cast<float*>(static_cast<char*>(workspace) + lse_bytes(a, c)) : nullptr;
    args.blocks = (int)c.blocks;
    args.splits = c.splits;
    args.tiles = c.tiles;
    const int64_t grid = c.blocks * args.groups * c.splits;
    if (grid >= (int64_t(1) << 24)) return DIVISION_ERANGE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (a.dt == DIVISION_BF16) return a.D <= 64 ? run<uint16_t, 64>(args, c, grid, st) : a.D <= 96 && !c.few ? run<uint16_t, 96>(args, c, grid, st) : run<uint16_t, 128>(args, c, grid, st);
    return a.D <= 32 ? run<float, 32>(args, c, grid, st) : a.D <= 64 ? run<float, 64>(args, c, grid, st) : a.D <= 96 ? run<float, 96>(args, c, grid, st) : run<float, 128>(args, c, grid, st);
}

}  // extern "C"
