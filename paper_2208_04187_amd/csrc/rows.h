// Included inside the unnamed namespaces of norm.hip, logprobs.hip and gradnorm.hip: rows of fp32 or bfloat16 elements in
// pieces of eight, reductions over lanes, launches.

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int kPiece = 8;                                   // elements a lane takes at a time: 16 bytes of bfloat16, 32 of fp32

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }
// two fp32 -> bfloat16 in one word, to nearest even, a NaN kept
__device__ __forceinline__ uint32_t bf16_pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2_t));
}

// Whole vectors at any element's address: of a type that says so, not byte by byte with memcpy, which the compiler took apart (four fp32 into a store of three and one of one: 513 x
// 32003 logits' gradient 30 us, 24 so).  PAST: the caches do not keep them.  Calls whose tensors are more than kCached together take that: what is read would not stay till the
// next one, and the last-level cache (256 MB) loses nothing that it would give.
constexpr int64_t kCached = int64_t(1) << 28;
template <typename V, bool PAST, typename T> __device__ __forceinline__ V load_vector(const T* p) {
    typedef V at_any_element __attribute__((aligned(alignof(T))));
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const at_any_element*>(p));
    else return *reinterpret_cast<const at_any_element*>(p);
}
template <bool PAST, typename T, typename V> __device__ __forceinline__ void store_vector(T* p, V q) {
    typedef V at_any_element __attribute__((aligned(alignof(T))));
    if constexpr (PAST) __builtin_nontemporal_store(q, reinterpret_cast<at_any_element*>(p));
    else *reinterpret_cast<at_any_element*>(p) = q;
}

__device__ __forceinline__ uint16_t bf16_of(float v) { return (uint16_t)bf16_pack2(v, 0.0f); }

// N elements of a row in a lane's registers: 4 or 8 of fp32 (float) or bfloat16 (uint16_t).  A row may start at any element: rows of an odd width do, and
// then no 16-byte access is aligned.  The machine takes such accesses of global memory (the ABI sets the unaligned mode).
template <typename T, int N> struct Some {
    static constexpr int kSize = N, kBytes = N * (int)sizeof(T);
    uint32_t w[kBytes / 4];

    __device__ __forceinline__ void fill(uint32_t word) {
#pragma unroll
        for (uint32_t& v : w) v = word;
    }
    __device__ __forceinline__ void zero() { fill(0); }
    template <bool PAST = false> __device__ __forceinline__ void load(const T* p) {
        if constexpr (kBytes == 8) {
            const u32x2 q = load_vector<u32x2, PAST>(p);
            w[0] = q.x; w[1] = q.y;
        } else {
#pragma unroll
            for (int k = 0; k < kBytes / 16; ++k) {
                const u32x4 q = load_vector<u32x4, PAST>(p + k * (16 / (int)sizeof(T)));
                w[4 * k] = q.x; w[4 * k + 1] = q.y; w[4 * k + 2] = q.z; w[4 * k + 3] = q.w;
            }
        }
    }
    // the elements lo .. hi - 1 alone, `word` beside them
    __device__ __forceinline__ void load(const T* p, int lo, int hi, uint32_t word = 0) {
        fill(word);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < lo || i >= hi) continue;
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[i]);
            else w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (uint32_t)p[i] << 16 : (w[i / 2] & 0xffff0000u) | p[i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return i & 1 ? __uint_as_float(w[i / 2] & 0xffff0000u) : bf16_value(w[i / 2]);
    }
    template <bool PAST = false> static __device__ __forceinline__ void store(T* p, const float* v) {
        uint32_t w[kBytes / 4];
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
            else w[i] = bf16_pack2(v[2 * i], v[2 * i + 1]);
        }
        if constexpr (kBytes == 8) {
            store_vector<PAST>(p, u32x2{w[0], w[1]});
        } else {
#pragma unroll
            for (int k = 0; k < kBytes / 16; ++k) store_vector<PAST>(p + k * (16 / (int)sizeof(T)), u32x4{w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]});
        }
    }
    static __device__ __forceinline__ void store(T* p, const float* v, int lo, int hi) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < lo || i >= hi) continue;
            if constexpr (sizeof(T) == 4) p[i] = v[i];
            else p[i] = bf16_of(v[i]);
        }
    }
};
template <typename T> using Piece = Some<T, kPiece>;
// Sixteen bytes: what an access of a lane moves.  (Eight elements of fp32 are two accesses, each of which leaves gaps between the lanes.)
template <typename T> using Unit = Some<T, 16 / (int)sizeof(T)>;

// The N elements of a row from column c of D on: whole, the row's last, or behind its end (zeros, nothing stored).  C: int where c + N fits it, else int64_t
template <typename S, bool PAST = false, typename T, typename C> __device__ __forceinline__ S load_some(const T* row, C c, C D) {
    S q;
    if (c + S::kSize <= D) q.template load<PAST>(row + c);
    else if (c < D) q.load(row + c, 0, (int)(D - c));
    else q.zero();
    return q;
}
template <typename S, bool PAST = false, typename T, typename C> __device__ __forceinline__ void store_some(T* row, C c, C D, const float* v) {
    if (c + S::kSize <= D) S::template store<PAST>(row + c, v);
    else if (c < D) S::store(row + c, v, 0, (int)(D - c));
}

// Reductions over aligned groups of lanes by DPP (no LDS, no waits): every lane gets the result.  Within 16 lanes the four steps pair each lane with
// its neighbour, the other pair of its quad, the mirrored half-row and the mirrored row; across rows through the permutes of 16 and 32 lanes.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
struct AddF { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); } };
struct MaxU { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; } };
struct MaxF { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); } };
// LANES: 4, 8, 16, 32 or 64; all lanes active
template <typename Op, int LANES> __device__ __forceinline__ uint32_t over_lanes(uint32_t v) {
    v = Op::of(v, dpp<kXor1>(v));
    v = Op::of(v, dpp<kXor2>(v));
    if constexpr (LANES >= 8) v = Op::of(v, dpp<kHalfMirror>(v));
    if constexpr (LANES >= 16) v = Op::of(v, dpp<kMirror>(v));
    if constexpr (LANES >= 32) v = Op::of(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    if constexpr (LANES >= 64) v = Op::of(v, (uint32_t)__shfl_xor((int)v, 32, 64));
    return v;
}
template <int LANES> __device__ __forceinline__ float sum_lanes(float v) { return __uint_as_float(over_lanes<AddF, LANES>(__float_as_uint(v))); }

// Which of a workgroup's rows, NT threads each, the thread works on; the same for all of a wavefront where it has one, and then in a scalar register: the
// row's addresses take no vector registers
template <int NT> __device__ __forceinline__ int row_of_thread() {
    if constexpr (NT >= 64) return __builtin_amdgcn_readfirstlane((int)threadIdx.x / NT);
    else return (int)threadIdx.x / NT;
}

// A value of a row over the NT threads that share it: NT up to 64 lanes of a wavefront, or whole wavefronts through `slots`, one per wavefront of the
// workgroup (which may hold several rows; all of it takes part).  One barrier: the next call but one may take the same slots again.
template <typename Op, int NT> __device__ __forceinline__ uint32_t over_row(uint32_t v, uint32_t* slots) {
    if constexpr (NT <= 64) {
        return over_lanes<Op, NT>(v);
    } else {
        constexpr int W = NT / 64;
        v = over_lanes<Op, 64>(v);
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        const uint32_t* own = slots + threadIdx.x / NT * W;
        uint32_t r = own[0];
#pragma unroll
        for (int i = 1; i < W; ++i) r = Op::of(r, own[i]);
        return r;
    }
}
template <int NT> __device__ __forceinline__ float row_sum(float v, uint32_t* slots) { return __uint_as_float(over_row<AddF, NT>(__float_as_uint(v), slots)); }
