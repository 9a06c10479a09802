// Rows of a token model's table, scaled, and the table's gradient, for AMD MI355X (gfx950).
//
//   out[t] = scale * table[ids[t]];   grad_table[v] = scale * sum of grad[t] over the tokens t with ids[t] = v
//
// The gradient's tokens are put in the order of (id, t) first, so that every row's sum is taken in the order of its tokens: no atomic touches a
// floating-point number.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "../../include/division.h"

namespace {
#include "rows.h"

constexpr int kThreads = 256;

// ------------------------------------------------------------------ lookup

struct LookupArgs {
    const int64_t* ids;
    const void* table;
    void* out;
    int64_t T, V, D, ignore;
    float scale;
    int each;                                               // pieces of a row
};
// A piece of sixteen bytes a lane; ids[t] behind the table is no token: its row is NaN.  Bound by memory and, in small calls, two trips to it: 2999 rows of 1155 in fp32 5.5 us = 5.0 TB/s (rows
// start at any element).
template <typename T, bool PAST> __global__ __launch_bounds__(kThreads) void lookup(LookupArgs a) {
    typedef Unit<T> U;
    const uint32_t e = blockIdx.x * kThreads + threadIdx.x, token = e / (uint32_t)a.each;       // below 2^32: a launch has no more threads
    if (token >= a.T) return;
    const int64_t t = token, c = (int64_t)(e - token * (uint32_t)a.each) * U::kSize, id = a.ids[t];
    float v[U::kSize];
    if (id >= 0 && id < a.V && id != a.ignore) {
        const U q = load_some<U>(static_cast<const T*>(a.table) + id * a.D, c, a.D);
#pragma unroll
        for (int i = 0; i < U::kSize; ++i) v[i] = q[i] * a.scale;
    } else {
#pragma unroll
        for (int i = 0; i < U::kSize; ++i) v[i] = id == a.ignore ? 0.0f : __uint_as_float(0x7fc00000u);
    }
    store_some<U, PAST>(static_cast<T*>(a.out) + t * a.D, c, a.D, v);
}

// ------------------------------------------------------------------ the tokens in the order of their ids

struct AddU { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a + b; } };
constexpr int kOrderThreads = 1024, kOrderWaves = kOrderThreads / 64, kMostRows = 512;       // rows of the table whose tokens a workgroup puts in order
constexpr int kKept = 16;                                   // ids of a thread that come at once

// Rows are dealt out to the workgroups like cards, since a tokenizer's frequent tokens have the lowest numbers: row k 2^bits + w of the table is row k of workgroup w, place w * rows + k of all.
// (16384 tokens whose frequencies fall as 1 / (number + 3): 25.5 us with neighbours in a workgroup, 12.6 so, and the rows' sums 32 and 24.)
struct Dealt {
    int bits;                                               // of the workgroups' number
    uint32_t rows;                                          // of a workgroup
    __host__ __device__ __forceinline__ uint32_t workgroups() const { return 1u << bits; }
    __host__ __device__ __forceinline__ uint32_t places() const { return rows << bits; }
    __device__ __forceinline__ uint32_t place(uint32_t row) const { return (row & (workgroups() - 1)) * rows + (row >> bits); }
    __device__ __forceinline__ uint32_t row(uint32_t place) const { return (place % rows << bits) + place / rows; }
};
struct OrderArgs {
    const int64_t* ids;
    uint32_t *order, *starts;                               // [T] tokens by (place of the id, number); [places + 1] where a place's begin
    int64_t V, ignore;
    uint32_t T;
    int bits;                                               // of a row's number among a workgroup's
    Dealt dealt;
};

// One launch instead of the passes of a sort.  Every workgroup reads all ids and keeps those of its rows; how many lie before its rows tells it where its tokens begin, so that workgroups need not wait for one another.  Each wavefront
// has an equal run of the tokens.  First they count: [row][wavefront].  The running sum over these numbers is where a wavefront's tokens of a row begin, and then each puts its own there,
// in their order.  Bound by its chain: 16384 tokens of 32768 rows, 256 workgroups, 10.5 us for even tokens, 13 for uneven ones: 2 until all workgroups have begun, 3 to 4 until all ids are sorted out
// (loaded one by one, 4 more), 1.3 for the running sum, 1 and more for putting tokens in their places.
__global__ __launch_bounds__(kOrderThreads) void order_tokens(OrderArgs a) {
    extern __shared__ uint32_t counts[];                    // [rows][kOrderWaves]
    __shared__ uint32_t sums[kOrderWaves], before;
    __shared__ uint16_t kept[kKept][kOrderThreads];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = (int)a.dealt.rows * kOrderWaves;
    const uint32_t run = (((a.T + kOrderWaves - 1) / kOrderWaves) + 63) & ~63u, first = wave * run, end = min(first + run, a.T);
    for (int e = threadIdx.x; e < n; e += kOrderThreads) counts[e] = 0;
    if (threadIdx.x == 0) before = 0;
    __syncthreads();
    constexpr uint32_t kNone = 0xffffu;                     // not of the workgroup's rows
    // of kKept times 64 tokens, whose ids come at once, behind the run's end zeros; `lower` counts those of workgroups before.  (By way of a bounded buffer and 32-bit comparisons: four wavefronts a SIMD do each of these instructions, and with
    // 64-bit addresses and comparisons they took half as long again as the trip to memory.)
    const uint32_t ignore = a.ignore >= 0 && a.ignore < a.V ? (uint32_t)a.ignore : 0xffffffffu;
    const auto rows_of = [&](uint32_t* to, uint32_t t, uint32_t& lower) {
        const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<int64_t*>(a.ids + t), 0, (int)((end - t < kKept * 64 ? end - t : kKept * 64) * 8), 0x00020000);
        const uint32_t there = end - t > (uint32_t)lane ? (end - t - lane + 63) / 64 : 0;
        u32x2 ids[kKept];
#pragma unroll
        for (int k = 0; k < kKept; ++k) ids[k] = __builtin_amdgcn_raw_buffer_load_b64(from, (k * 64 + lane) * 8, 0, 0);
#pragma unroll
        for (int k = 0; k < kKept; ++k) {
            const uint32_t id = ids[k].x;
            const bool one = ((uint32_t)k < there) & (ids[k].y == 0) & (id < (uint32_t)a.V) & (id != ignore);
            const uint32_t w = one ? id & (a.dealt.workgroups() - 1) : 0xffffffffu, row = id >> a.dealt.bits;
            to[k] = w == blockIdx.x ? row : kNone;
            lower += w < blockIdx.x ? 1u : 0u;
        }
    };
    uint32_t less = 0;
    for (uint32_t t = first; t < end; t += kKept * 64) {
        uint32_t rows[kKept];
        rows_of(rows, t, less);
#pragma unroll
        for (int k = 0; k < kKept; ++k) {
            if (rows[k] != kNone) atomicAdd(&counts[rows[k] * kOrderWaves + wave], 1u);
            if (t == first) kept[k][threadIdx.x] = (uint16_t)rows[k];
        }
    }
    less = over_lanes<AddU, 64>(less);
    if (lane == 0) atomicAdd(&before, less);
    __syncthreads();
    // running sum over all numbers: a run of them a thread
    const int each = (n + kOrderThreads - 1) / kOrderThreads, from = min((int)threadIdx.x * each, n), to = min(from + each, n);
    uint32_t own = 0;
    for (int e = from; e < to; ++e) own += counts[e];
    uint32_t upto = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = (uint32_t)__shfl_up((int)upto, o, 64);
        if (lane >= o) upto += v;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t at = before + upto - own + over_lanes<AddU, kOrderWaves>((lane & (kOrderWaves - 1)) < wave ? sums[lane & (kOrderWaves - 1)] : 0u);
    for (int e = from; e < to; ++e) {
        const uint32_t c = counts[e];
        counts[e] = at;
        if (e % kOrderWaves == 0) a.starts[blockIdx.x * a.dealt.rows + e / kOrderWaves] = at;
        at += c;
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == kOrderThreads - 1) a.starts[a.dealt.places()] = at;
    __syncthreads();
    // A row's tokens among the wavefront's 64: where there is one row or two, which is most often, one after the other; the lanes of more rows find their likes by the rows' bits.  (All by their bits:
    // 6 us more for 16384 tokens of 32768; all one after the other: a third of a microsecond for each row.)  The wavefront's own counter is moved on by one lane with an atomic, since the next
    // that reads it is another's.
    const auto place = [&](uint32_t row, uint32_t t) {
        const uint64_t below = (1ull << lane) - 1;
        uint64_t left = __ballot(row != kNone);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (!left) return;
            const int leader = __builtin_ctzll(left);
            const uint32_t theirs = (uint32_t)__builtin_amdgcn_readlane((int)row, leader);
            const uint64_t same = __ballot(row == theirs);
            uint32_t begin = 0;
            if (lane == leader) begin = atomicAdd(&counts[theirs * kOrderWaves + wave], (uint32_t)__builtin_popcountll(same));
            begin = (uint32_t)__builtin_amdgcn_readlane((int)begin, leader);
            if (row == theirs) a.order[begin + __builtin_popcountll(same & below)] = t;
            left &= ~same;
        }
        if (!left) return;
        const bool mine = left >> lane & 1;
        uint64_t same = left;
        for (int bit = 0; bit < a.bits; ++bit) {
            const uint64_t set = __ballot(row >> bit & 1);
            same &= row >> bit & 1 ? set : ~set;
        }
        const int leader = mine ? __builtin_ctzll(same) : 0;
        uint32_t begin = 0;
        if (mine && lane == leader) begin = atomicAdd(&counts[row * kOrderWaves + wave], (uint32_t)__builtin_popcountll(same));
        begin = (uint32_t)__shfl((int)begin, leader, 64);
        if (mine) a.order[begin + __builtin_popcountll(same & below)] = t;
    };
    // (One round after another, not unrolled: sixteen copies of it take longer to come from memory than to run.)
    for (uint32_t t = first; t < end; t += kKept * 64) {
        if (t != first) {
            uint32_t rows[kKept];
            rows_of(rows, t, less);
#pragma unroll
            for (int k = 0; k < kKept; ++k) kept[k][threadIdx.x] = (uint16_t)rows[k];
        }
#pragma unroll 1
        for (int k = 0; k < kKept; ++k) place(kept[k][threadIdx.x], t + k * 64 + lane);
    }
}

// ------------------------------------------------------------------ the rows' sums

struct SumArgs {
    const void* grad;
    const int64_t* ids;
    const uint32_t *order, *starts;
    Dealt dealt;
    float* parts;                                           // [parts of the sorted tokens][2][D]: of the row that began before the part, of the one that begins in it
    void* out;
    int64_t stride, V, D;
    uint32_t T, part;                                       // part: tokens that a wavefront adds up at most; a row of more is added up in parts
    float scale;
    int add, columns, rows, whole;                          // columns: pieces of 64 * kSize * P elements of a row; whole: no row ends within a vector
    int64_t count;                                          // parts of the tokens, where there are more than one's
};

// P vectors a lane of a row's columns, 64 lanes' vectors one behind the other
template <typename T, int P> struct Row {
    typedef Unit<T> U;
    float v[P][U::kSize];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < U::kSize; ++i) v[p][i] = 0.0f;
    }
    // adds tokens order[from .. to - 1]; c: a column.  64 tokens' numbers come at once, a lane each, their rows several at a time.
    __device__ __forceinline__ void add(const SumArgs& a, uint32_t from, uint32_t to, int64_t c) {
        if (a.whole) add_of<true>(a, from, to, c);
        else add_of<false>(a, from, to, c);
    }
    // WHOLE: rows are whole vectors.  Lanes behind the last column take the first one's, so that no load waits for a branch
    template <bool WHOLE> __device__ __forceinline__ void add_of(const SumArgs& a, uint32_t from, uint32_t to, int64_t c) {
        int64_t cs[P];
#pragma unroll
        for (int p = 0; p < P; ++p) cs[p] = WHOLE && c + p * 64 * U::kSize >= a.D ? 0 : c + p * 64 * U::kSize;
        const auto load = [&](U& q, const T* row, int p) {
            if constexpr (WHOLE) q.load(row + cs[p]);
            else q = load_some<U>(row, cs[p], a.D);
        };
        constexpr int kAtOnce = P == 1 ? 8 : 4;
        const T* grad = static_cast<const T*>(a.grad);
        const uint32_t lane = threadIdx.x & 63;
        for (uint32_t k = from; k < to; k += 64) {
            const int n = (int)min(to - k, 64u);
            const int tokens = (int)a.order[min(k + lane, to - 1)];
            int j = 0;
            for (; j + kAtOnce <= n; j += kAtOnce) {
                U q[kAtOnce][P];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const T* row = grad + (int64_t)(uint32_t)__builtin_amdgcn_readlane(tokens, j + u) * a.stride;
#pragma unroll
                    for (int p = 0; p < P; ++p) load(q[u][p], row, p);
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int i = 0; i < U::kSize; ++i) v[p][i] += q[u][p][i];
            }
            // the last ones all at once too: rows that are none count for nothing
            if (j < n) {
                U q[kAtOnce - 1][P];
#pragma unroll
                for (int u = 0; u < kAtOnce - 1; ++u) {
                    const T* row = grad + (int64_t)(uint32_t)__builtin_amdgcn_readlane(tokens, min(j + u, n - 1)) * a.stride;
#pragma unroll
                    for (int p = 0; p < P; ++p) load(q[u][p], row, p);
                }
#pragma unroll
                for (int u = 0; u < kAtOnce - 1; ++u) {
                    if (j + u >= n) break;
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int i = 0; i < U::kSize; ++i) v[p][i] += q[u][p][i];
                }
            }
        }
    }
};

// A row's sum goes out: scaled, rounded, added to what is there
template <typename T, typename O, int P> __device__ __forceinline__ void put_row(const SumArgs& a, int64_t row, int64_t c, Row<T, P>& sum) {
    typedef Unit<T> U;
    typedef Some<O, U::kSize> Out;
    O* out = static_cast<O*>(a.out) + row * a.D;
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int i = 0; i < U::kSize; ++i) sum.v[p][i] *= a.scale;
        if (a.add) {
            const Out q = load_some<Out>(out, c + p * 64 * U::kSize, a.D);
#pragma unroll
            for (int i = 0; i < U::kSize; ++i) sum.v[p][i] += q[i];
        }
        store_some<Out>(out, c + p * 64 * U::kSize, a.D, sum.v[p]);
    }
}

// Parts of rows of many tokens: a wavefront has `part` sorted tokens and a piece of the columns.  Of such rows at most two have tokens among them.
template <typename T, int P> __device__ __forceinline__ void sum_part(const SumArgs& a, uint32_t part, int64_t c) {
    typedef Unit<T> U;
    const uint32_t begin = part * a.part, total = a.starts[a.dealt.places()];
    if (begin >= total) return;
    const uint32_t end = min(begin + a.part, total);
    const uint32_t places[2] = {a.dealt.place((uint32_t)a.ids[a.order[begin]]), a.dealt.place((uint32_t)a.ids[a.order[end - 1]])};
    for (int k = 0; k < 2; ++k) {
        if (k && places[1] == places[0]) break;
        const uint32_t from = a.starts[places[k]], to = a.starts[places[k] + 1];
        if (to - from <= a.part) continue;
        Row<T, P> sum;
        sum.zero();
        sum.add(a, max(from, begin), min(to, end), c);
        float* out = a.parts + ((int64_t)part * 2 + (from >= begin)) * a.D;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < U::kSize; i += 4) store_some<Unit<float>>(out, c + p * 64 * U::kSize + i, a.D, sum.v[p] + i);
    }
}

// The table's gradient: the first wavefronts have parts of rows of many tokens, each of the others kRows rows (one where there are not wavefronts enough for all SIMDs otherwise), whose tokens lie
// one behind the other in the order; all a piece of the columns.  No row is written twice, rows without a token get their zeros here.  Bound by memory and the longest chain, three dependent loads
// before the first row: 16384 tokens of 32768 rows of 1024 in bfloat16 18 us (100 MB), 24 where tokens are as uneven as 1 / (number + 3).
constexpr int kRows = 4;
template <typename T, typename O, int P> __global__ __launch_bounds__(kThreads) void sum_tokens(SumArgs a) {
    typedef Unit<T> U;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), which = item / a.columns;
    const int64_t c = ((item - which * a.columns) * 64 * P + (threadIdx.x & 63)) * U::kSize;
    if (which < a.count) {
        sum_part<T, P>(a, (uint32_t)which, c);
        return;
    }
    const int64_t place0 = (which - a.count) * a.rows, places = a.dealt.places();
    if (place0 >= places) return;
    uint32_t starts[kRows + 1];
#pragma unroll
    for (int r = 0; r <= kRows; ++r) starts[r] = a.starts[place0 + r < places ? place0 + r : places];
    for (int r = 0; r < a.rows; ++r) {
        if (place0 + r >= places) return;
        const int64_t row = a.dealt.row((uint32_t)(place0 + r));
        const uint32_t n = starts[r + 1] - starts[r];
        if (row >= a.V || n > a.part || (a.add && n == 0)) continue;
        Row<T, P> sum;
        sum.zero();
        sum.add(a, starts[r], starts[r + 1], c);
        put_row<T, O, P>(a, row, c, sum);
    }
}

// The rows of many tokens, from their parts: the workgroup of the part that such a row begins in has it, a wavefront every fourth part.  Bound by the same chain: 7 us.
template <typename T, typename O, int P> __global__ __launch_bounds__(kThreads) void join_rows(SumArgs a) {
    typedef Unit<T> U;
    constexpr int kWaves = kThreads / 64;
    __shared__ float sums[kWaves - 1][P * U::kSize][64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x & 63;
    const uint32_t part = blockIdx.x / a.columns, begin = part * a.part, total = a.starts[a.dealt.places()];
    if (begin >= total) return;
    const int64_t row = a.ids[a.order[min(begin + a.part, total) - 1]];             // it goes on behind the part
    const uint32_t place = a.dealt.place((uint32_t)row), from = a.starts[place], to = a.starts[place + 1];
    if (to - from <= a.part || from < begin) return;
    const int64_t c = ((int64_t)(blockIdx.x - part * a.columns) * 64 * P + lane) * U::kSize;
    Row<T, P> sum;
    sum.zero();
    const uint32_t last = (to - 1) / a.part;
#pragma unroll 4
    for (uint32_t k = part + wave; k <= last; k += kWaves) {
        const float* q = a.parts + ((int64_t)k * 2 + (k == part)) * a.D;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < U::kSize; i += 4) {
                const Unit<float> u = load_some<Unit<float>>(q, c + p * 64 * U::kSize + i, a.D);
#pragma unroll
                for (int n = 0; n < 4; ++n) sum.v[p][i + n] += u[n];
            }
    }
    if (wave) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < U::kSize; ++i) sums[wave - 1][p * U::kSize + i][lane] = sum.v[p][i];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < U::kSize; ++i) sum.v[p][i] += sums[w][p * U::kSize + i][lane];
    put_row<T, O, P>(a, row, c, sum);
}

// ------------------------------------------------------------------ host side

#include "launch.h"
constexpr int64_t kMostWorkgroups = int64_t(1) << 24, kMostTokens = int64_t(1) << 31, kMostElements = int64_t(1) << 40;

// tokens of a part: few enough that one row's keep many wavefronts busy, and no more than 2048 parts, which the row's own adds up one after the other
uint32_t part_of(int64_t T) {
    uint32_t n = 32;
    while (T / n > 2048) n *= 2;
    return n;
}
// the workspace: order, starts, parts
struct Places { size_t order, starts, parts, bytes; Dealt dealt; };
Places places_of(int64_t T, int64_t V, int64_t D) {
    Places p;
    p.dealt.bits = 0;                                       // 256 workgroups, one a CU, since each reads all ids; fewer for fewer rows, more where they would have more than kMostRows
    while (((int64_t)1 << p.dealt.bits) < V && (p.dealt.bits < 8 || (V >> p.dealt.bits) >= kMostRows)) ++p.dealt.bits;
    p.dealt.rows = (uint32_t)((V + p.dealt.workgroups() - 1) >> p.dealt.bits);
    p.order = 0;
    p.starts = (size_t)(T * 4 + 15) / 16 * 16;
    p.parts = p.starts + ((size_t)p.dealt.places() * 4 + 4 + 15) / 16 * 16;
    p.bytes = p.parts + (T > part_of(T) ? (size_t)((T + part_of(T) - 1) / part_of(T)) * 2 * D * 4 : 0);
    return p;
}
int check_sizes(int64_t T, int64_t V, int64_t D) {
    if (T < 0 || V < 1 || D < 1) return DIVISION_EINVAL;
    if (T >= kMostTokens || V >= kMostTokens || D >= kMostTokens || (T > 0 && D > kMostElements / T) || D > kMostElements / V) return DIVISION_ERANGE;
    return DIVISION_OK;
}

}  // namespace

extern "C" {

int division_embedding(const int64_t* ids, int64_t T, const void* table, int64_t V, int64_t D, division_dtype dt, float scale, int64_t ignore_index, void* out, void* hip_stream) {
    if (!type_ok(dt)) return DIVISION_EINVAL;
    CHECKED(check_sizes(T, V, D));
    if (T == 0) return DIVISION_OK;
    if (!ids || !table || !out) return DIVISION_EINVAL;
    if (!aligned(ids, 8) || !aligned(table, size_of(dt)) || !aligned(out, size_of(dt))) return DIVISION_EALIGN;
    const int64_t size = 16 / size_of(dt), each = (D + size - 1) / size, grid = (T * each + kThreads - 1) / kThreads;
    if (grid >= kMostWorkgroups) return DIVISION_ERANGE;
    const LookupArgs a{ids, table, out, T, V, D, ignore_index, scale, (int)each};
    const bool past = T * D * (int64_t)size_of(dt) > kCached;
    void (*kernel)(LookupArgs) = dt == DIVISION_BF16 ? (past ? lookup<uint16_t, true> : lookup<uint16_t, false>) : past ? lookup<float, true> : lookup<float, false>;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), a);
    return launched();
}

size_t division_embedding_backward_workspace(int64_t T, int64_t V, int64_t D) { return check_sizes(T, V, D) == DIVISION_OK ? places_of(T, V, D).bytes : 0; }

int division_embedding_backward(const division_embedding_back* back, void* hip_stream) {
    if (!back) return DIVISION_EINVAL;
    const division_embedding_back& b = *back;
    if (!type_ok(b.dt) || !type_ok(b.table_dt) || b.grad_stride < 0 || (b.add != 0 && b.add != 1)) return DIVISION_EINVAL;
    CHECKED(check_sizes(b.T, b.V, b.D));
    if (b.T > 0 && b.grad_stride > kMostElements / b.T) return DIVISION_ERANGE;
    if (!b.grad_table || !b.workspace || (b.T > 0 && (!b.grad || !b.ids))) return DIVISION_EINVAL;
    if (!aligned(b.grad, size_of(b.dt)) || !aligned(b.ids, 8) || !aligned(b.grad_table, size_of(b.table_dt)) || !aligned(b.workspace, 16)) return DIVISION_EALIGN;
    const Places at = places_of(b.T, b.V, b.D);
    if (b.workspace_bytes < at.bytes) return DIVISION_ESIZE;
    char* ws = static_cast<char*>(b.workspace);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const Dealt& dealt = at.dealt;
    if ((int64_t)dealt.workgroups() * kOrderThreads >= (int64_t(1) << 32)) return DIVISION_ERANGE;
    OrderArgs o{b.ids, reinterpret_cast<uint32_t*>(ws + at.order), reinterpret_cast<uint32_t*>(ws + at.starts), b.V, b.ignore_index, (uint32_t)b.T, 0, dealt};
    while ((1u << o.bits) < dealt.rows) ++o.bits;
    const uint32_t part = part_of(b.T);
    SumArgs s{b.grad, b.ids, o.order, o.starts, dealt, reinterpret_cast<float*>(ws + at.parts), b.grad_table, b.grad_stride, b.V, b.D, (uint32_t)b.T, part, b.scale, b.add, 0, 0, b.D % (16 / (int64_t)size_of(b.dt)) == 0, 0};
    const bool wide = b.D > 64 * (int64_t)(16 / size_of(b.dt));
    const int64_t each = 64 * (int64_t)(16 / size_of(b.dt)) * (wide ? 2 : 1), columns = (b.D + each - 1) / each;
    s.columns = (int)columns;
    s.count = b.T > part ? (b.T + part - 1) / part : 0;
    s.rows = b.V * columns < 8192 * kRows ? 1 : kRows;
    const int64_t joins = s.count * columns, grid = ((s.count + ((int64_t)dealt.places() + s.rows - 1) / s.rows) * columns + 3) / 4;
    if (grid >= kMostWorkgroups || joins >= kMostWorkgroups) return DIVISION_ERANGE;
    hipLaunchKernelGGL(order_tokens, dim3(dealt.workgroups()), dim3(kOrderThreads), (size_t)dealt.rows * kOrderWaves * 4, st, o);
    CHECKED(launched());
    const bool half = b.dt == DIVISION_BF16;
    void (*sum)(SumArgs);
    void (*join)(SumArgs);
#define OF_TYPES(T, O) sum = wide ? sum_tokens<T, O, 2> : sum_tokens<T, O, 1>; join = wide ? join_rows<T, O, 2> : join_rows<T, O, 1>
    if (b.table_dt == DIVISION_BF16) {
        if (half) { OF_TYPES(uint16_t, uint16_t); } else { OF_TYPES(float, uint16_t); }
    } else {
        if (half) { OF_TYPES(uint16_t, float); } else { OF_TYPES(float, float); }
    }
#undef OF_TYPES
    hipLaunchKernelGGL(sum, dim3((uint32_t)grid), dim3(kThreads), 0, st, s);
    CHECKED(launched());
    if (!s.count) return DIVISION_OK;
    hipLaunchKernelGGL(join, dim3((uint32_t)joins), dim3(kThreads), 0, st, s);
    return launched();
}

}  // extern "C"
