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

// Accesses that the caches do not keep.  Calls whose tensors are more than kCached together take them: what is read would not stay till the next
// one, and the last-level cache (256 MB) loses nothing that it would give.
constexpr int64_t kCached = int64_t(1) << 28;
template <typename V, typename T> __device__ __forceinline__ V load_past(const T* p) {
    typedef V at_any_element __attribute__((aligned(alignof(T))));
    return __builtin_nontemporal_load(reinterpret_cast<const at_any_element*>(p));
}
template <typename T, typename V> __device__ __forceinline__ void store_past(T* p, V q) {
    typedef V at_any_element __attribute__((aligned(alignof(T))));
    __builtin_nontemporal_store(q, reinterpret_cast<at_any_element*>(p));
}

// Element types: fp32 as float, bfloat16 as uint16_t.  A row may start at any element: rows of an odd width do, and then no
// 16-byte access is aligned.  The machine takes such accesses of global memory (the ABI sets the unaligned mode); memcpy says so to the compiler, which
// keeps them whole.
template <typename T> struct Piece;
template <> struct Piece<float> {
    u32x4 w[2];
    template <bool PAST = false> __device__ __forceinline__ void load(const float* p) {
        if constexpr (PAST) { w[0] = load_past<u32x4>(p); w[1] = load_past<u32x4>(p + 4); }
        else __builtin_memcpy(w, p, 32);
    }
    // its elements lo .. hi - 1 alone, zeros beside them
    __device__ __forceinline__ void load(const float* p, int lo, int hi) {
        uint32_t* e = reinterpret_cast<uint32_t*>(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i >= lo && i < hi ? __float_as_uint(p[i]) : 0u;
    }
    __device__ __forceinline__ void zero() { w[0] = u32x4{0, 0, 0, 0}; w[1] = w[0]; }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(w[i / 4][i % 4]); }
    template <bool PAST = false> static __device__ __forceinline__ void store(float* p, const float* v) {
        u32x4 q[2];
        __builtin_memcpy(q, v, 32);
        if constexpr (PAST) { store_past(p, q[0]); store_past(p + 4, q[1]); }
        else __builtin_memcpy(p, q, 32);
    }
    static __device__ __forceinline__ void store(float* p, const float* v, int lo, int hi) {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i >= lo && i < hi) p[i] = v[i];
    }
};
template <> struct Piece<uint16_t> {
    u32x4 w;
    template <bool PAST = false> __device__ __forceinline__ void load(const uint16_t* p) {
        if constexpr (PAST) w = load_past<u32x4>(p);
        else __builtin_memcpy(&w, p, 16);
    }
    __device__ __forceinline__ void load(const uint16_t* p, int lo, int hi) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t even = 2 * i >= lo && 2 * i < hi ? p[2 * i] : 0u, odd = 2 * i + 1 >= lo && 2 * i + 1 < hi ? p[2 * i + 1] : 0u;
            w[i] = even | odd << 16;
        }
    }
    __device__ __forceinline__ void zero() { w = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ float operator[](int i) const { return i & 1 ? __uint_as_float(w[i / 2] & 0xffff0000u) : bf16_value(w[i / 2]); }
    static __device__ __forceinline__ u32x4 packed(const float* v) {
        return u32x4{bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3]), bf16_pack2(v[4], v[5]), bf16_pack2(v[6], v[7])};
    }
    template <bool PAST = false> static __device__ __forceinline__ void store(uint16_t* p, const float* v) {
        const u32x4 q = packed(v);
        if constexpr (PAST) store_past(p, q);
        else __builtin_memcpy(p, &q, 16);
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float* v, int lo, int hi) {
        const u32x4 q = packed(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i >= lo && i < hi) p[i] = (uint16_t)(q[i / 2] >> (i & 1 ? 16 : 0));
    }
};
// The piece of a row that starts at column c of D: whole, the row's last, or behind its end (zeros, nothing stored).  C: int where c + 8 fits it, else int64_t
template <bool PAST = false, typename T, typename C> __device__ __forceinline__ Piece<T> load_piece(const T* row, C c, C D) {
    Piece<T> q;
    if (c + kPiece <= D) q.template load<PAST>(row + c);
    else if (c < D) q.load(row + c, 0, (int)(D - c));
    else q.zero();
    return q;
}
template <bool PAST = false, typename T, typename C> __device__ __forceinline__ void store_piece(T* row, C c, C D, const float* v) {
    if (c + kPiece <= D) Piece<T>::template store<PAST>(row + c, v);
    else if (c < D) Piece<T>::store(row + c, v, 0, (int)(D - c));
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
