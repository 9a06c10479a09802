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
// A piece of sixteen bytes a lane; ids[t] behind the table is no token: its row is NaN.
template <typename T, bool PAST> __global__ __launch_bounds__(kThreads) void lookup(LookupArgs a) {
    typedef Unit<T> U;
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x, t = e / a.each;
    if (t >= a.T) return;
    const int64_t c = (e - t * a.each) * U::kSize, id = a.ids[t];
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

constexpr int kOrderThreads = 1024, kOrderWaves = kOrderThreads / 64, kMostRows = 512;       // rows of the table whose tokens a workgroup puts in order

struct OrderArgs {
    const int64_t* ids;
    uint32_t *order, *starts;                               // [T] tokens by (id, number); [V + 1] where a row's begin
    int64_t V, ignore;
    uint32_t T;
    int rows;                                               // of a workgroup
};

// Every workgroup reads all ids and keeps those of its rows; how many lie before its rows tells it where its tokens begin, so that workgroups need not wait for one another.  Each wavefront
// has an equal run of the tokens.  First they count: [row][wavefront].  The running sum over these numbers is where a wavefront's tokens of a row begin, and then each puts its own there,
// in their order.  T ids are read twice by each workgroup, from the caches.
__global__ __launch_bounds__(kOrderThreads) void order_tokens(OrderArgs a) {
    extern __shared__ uint32_t counts[];                    // [rows][kOrderWaves]
    __shared__ uint32_t sums[kOrderWaves], before;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.rows * kOrderWaves;
    const int64_t lo = (int64_t)blockIdx.x * a.rows;
    const uint32_t rows = (uint32_t)(a.V - lo < a.rows ? a.V - lo : a.rows);
    const uint32_t run = (((a.T + kOrderWaves - 1) / kOrderWaves) + 63) & ~63u, first = wave * run, end = min(first + run, a.T);
    for (int e = threadIdx.x; e < n; e += kOrderThreads) counts[e] = 0;
    if (threadIdx.x == 0) before = 0;
    __syncthreads();
    uint32_t less = 0;
    for (uint32_t t = first + lane; t < end; t += 64) {
        const int64_t id = a.ids[t];
        if (id < 0 || id >= a.V || id == a.ignore) continue;
        if (id < lo) ++less;
        else if (id - lo < rows) atomicAdd(&counts[(uint32_t)(id - lo) * kOrderWaves + wave], 1u);
    }
    atomicAdd(&before, less);
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
    uint32_t at = before + upto - own;
    for (int w = 0; w < wave; ++w) at += sums[w];
    for (int e = from; e < to; ++e) {
        const uint32_t c = counts[e];
        counts[e] = at;
        if (e % kOrderWaves == 0 && (uint32_t)(e / kOrderWaves) < rows) a.starts[lo + e / kOrderWaves] = at;
        at += c;
    }
    if (lo + rows == a.V && threadIdx.x == kOrderThreads - 1) a.starts[a.V] = at;
    __syncthreads();
    for (uint32_t t0 = first; t0 < end; t0 += 64) {
        const uint32_t t = t0 + lane;
        const int64_t id = t < end ? a.ids[t] : -1;
        const bool mine = id >= lo && id - lo < rows && id != a.ignore;
        const uint32_t row = mine ? (uint32_t)(id - lo) : 0xffffffffu;
        uint64_t left = __ballot(mine);
        while (left) {                                      // the tokens of one row at a time
            const int leader = __builtin_ctzll(left);
            const uint32_t theirs = (uint32_t)__builtin_amdgcn_readlane((int)row, leader);
            const uint64_t same = __ballot(row == theirs);
            const uint32_t begin = counts[theirs * kOrderWaves + wave];
            if (row == theirs) a.order[begin + __builtin_popcountll(same & ((1ull << lane) - 1))] = t;
            if (lane == leader) counts[theirs * kOrderWaves + wave] = begin + __builtin_popcountll(same);
            left &= ~same;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // the next token of this row may be another lane's
        }
    }
}

// ------------------------------------------------------------------ the rows' sums

constexpr int kMany = 128;                                  // a row of more tokens is added up by several wavefronts, a part of so many tokens each

struct SumArgs {
    const void* grad;
    const int64_t* ids;
    const uint32_t *order, *starts;
    float* parts;                                           // [parts of the sorted tokens][2][D]: of the row that begins before the part, of the one that ends behind it
    void* out;
    int64_t stride, V, D;
    uint32_t T;
    float scale;
    int add, columns;                                       // columns: pieces of 512 elements (bfloat16) or 256 of a row
};

// C elements a lane of the sum over tokens order[from .. to - 1], four at a time on their way
template <typename T> __device__ __forceinline__ void sum_rows(const SumArgs& a, uint32_t from, uint32_t to, int64_t c, float* v) {
    typedef Unit<T> U;
    const T* grad = static_cast<const T*>(a.grad);
#pragma unroll
    for (int i = 0; i < U::kSize; ++i) v[i] = 0.0f;
    uint32_t k = from;
    for (; k + 4 <= to; k += 4) {
        U q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = load_some<U>(grad + (int64_t)a.order[k + u] * a.stride, c, a.D);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < U::kSize; ++i) v[i] += q[u][i];
    }
    for (; k < to; ++k) {
        const U q = load_some<U>(grad + (int64_t)a.order[k] * a.stride, c, a.D);
#pragma unroll
        for (int i = 0; i < U::kSize; ++i) v[i] += q[i];
    }
}

// Parts of rows of many tokens: a wavefront has kMany sorted tokens and a piece of the columns.  At most two such rows have tokens among them.
template <typename T> __global__ __launch_bounds__(kThreads) void sum_parts(SumArgs a) {
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const uint32_t part = (uint32_t)(item / a.columns), begin = part * kMany, total = a.starts[a.V];
    if (begin >= total) return;
    const uint32_t end = min(begin + kMany, total);
    const int64_t c = ((item % a.columns) * 64 + (threadIdx.x & 63)) * Unit<T>::kSize;
    const int64_t rows[2] = {a.ids[a.order[begin]], a.ids[a.order[end - 1]]};
    for (int k = 0; k < 2; ++k) {
        if (k && rows[1] == rows[0]) break;
        const uint32_t from = a.starts[rows[k]], to = a.starts[rows[k] + 1];
        if (to - from <= kMany) continue;
        float v[Unit<T>::kSize];
        sum_rows<T>(a, max(from, begin), min(to, end), c, v);
        // the second place: rows that begin in this part
        store_some<Unit<float>>(a.parts + ((int64_t)part * 2 + (from > begin)) * a.D, c, a.D, v);
        if constexpr (sizeof(T) == 2) store_some<Unit<float>>(a.parts + ((int64_t)part * 2 + (from > begin)) * a.D, c + 4, a.D, v + 4);
    }
}

// The table's gradient: a wavefront has a row and a piece of the columns.
template <typename T, typename O> __global__ __launch_bounds__(kThreads) void sum_tokens(SumArgs a) {
    typedef Unit<T> U;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64, row = item / a.columns;
    if (row >= a.V) return;
    const int64_t c = ((item % a.columns) * 64 + (threadIdx.x & 63)) * U::kSize;
    const uint32_t from = (uint32_t)__builtin_amdgcn_readfirstlane((int)a.starts[row]), to = (uint32_t)__builtin_amdgcn_readfirstlane((int)a.starts[row + 1]);
    if (a.add && from == to) return;
    float v[U::kSize];
    if (to - from <= kMany) {
        sum_rows<T>(a, from, to, c, v);
    } else {
#pragma unroll
        for (int i = 0; i < U::kSize; ++i) v[i] = 0.0f;
        for (uint32_t part = from / kMany; part <= (to - 1) / kMany; ++part) {
            const float* p = a.parts + ((int64_t)part * 2 + (from > part * kMany)) * a.D;
#pragma unroll
            for (int i = 0; i < U::kSize; i += 4) {
                const Unit<float> q = load_some<Unit<float>>(p, c + i, a.D);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i + k] += q[k];
            }
        }
    }
    O* out = static_cast<O*>(a.out) + row * a.D;
    typedef Some<O, U::kSize> Out;
#pragma unroll
    for (int i = 0; i < U::kSize; ++i) v[i] *= a.scale;
    if (a.add) {
        const Out q = load_some<Out>(out, c, a.D);
#pragma unroll
        for (int i = 0; i < U::kSize; ++i) v[i] += q[i];
    }
    store_some<Out>(out, c, a.D, v);
}

// ------------------------------------------------------------------ host side

bool type_ok(division_dtype dt) { return dt == DIVISION_F32 || dt == DIVISION_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? DIVISION_OK : DIVISION_EHIP; }
#define CHECKED(call) do { const int rc_ = (call); if (rc_ != DIVISION_OK) return rc_; } while (0)
size_t size_of(division_dtype dt) { return dt == DIVISION_BF16 ? 2 : 4; }
constexpr int64_t kMostWorkgroups = int64_t(1) << 24, kMostTokens = int64_t(1) << 31, kMostElements = int64_t(1) << 40;

// the workspace: order, starts, parts
struct Places { size_t order, starts, parts, bytes; };
Places places_of(int64_t T, int64_t V, int64_t D) {
    Places p;
    p.order = 0;
    p.starts = (size_t)(T * 4 + 15) / 16 * 16;
    p.parts = p.starts + (size_t)((V + 1) * 4 + 15) / 16 * 16;
    p.bytes = p.parts + (T > kMany ? (size_t)((T + kMany - 1) / kMany) * 2 * D * 4 : 0);
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
    OrderArgs o{b.ids, reinterpret_cast<uint32_t*>(ws + at.order), reinterpret_cast<uint32_t*>(ws + at.starts), b.V, b.ignore_index, (uint32_t)b.T, 0};
    // two workgroups a CU at most, a row each at least
    int64_t rows = (b.V + 511) / 512;
    if (rows > kMostRows) rows = kMostRows;
    o.rows = (int)rows;
    const int64_t workgroups = (b.V + rows - 1) / rows;
    if (workgroups * kOrderThreads >= (int64_t(1) << 32)) return DIVISION_ERANGE;
    const int64_t size = 16 / size_of(b.dt), columns = (b.D + 64 * size - 1) / (64 * size);
    const int64_t parts = ((b.T + kMany - 1) / kMany * columns + 3) / 4, grid = (b.V * columns + 3) / 4;
    if (parts >= kMostWorkgroups || grid >= kMostWorkgroups) return DIVISION_ERANGE;
    hipLaunchKernelGGL(order_tokens, dim3((uint32_t)workgroups), dim3(kOrderThreads), (size_t)rows * kOrderWaves * 4, st, o);
    CHECKED(launched());
    const SumArgs s{b.grad, b.ids, o.order, o.starts, reinterpret_cast<float*>(ws + at.parts), b.grad_table, b.grad_stride, b.V, b.D, (uint32_t)b.T, b.scale, b.add, (int)columns};
    if (b.T > kMany) {
        void (*kernel)(SumArgs) = b.dt == DIVISION_BF16 ? sum_parts<uint16_t> : sum_parts<float>;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)parts), dim3(kThreads), 0, st, s);
        CHECKED(launched());
    }
    void (*kernel)(SumArgs) = b.dt == DIVISION_BF16 ? (b.table_dt == DIVISION_BF16 ? sum_tokens<uint16_t, uint16_t> : sum_tokens<uint16_t, float>)
                              : b.table_dt == DIVISION_BF16 ? sum_tokens<float, uint16_t> : sum_tokens<float, float>;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(kThreads), 0, st, s);
    return launched();
}

}  // extern "C"
