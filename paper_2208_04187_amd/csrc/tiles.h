// Included inside the unnamed namespaces of attention.hip and attention_back.hip: tiles of rows in the local memory, matrix products of them, who sees whom.
//
// A product's 32 x 32 block is held as the matrix instruction leaves it: lane l has column l % 32, and of it the rows 8 (i / 4) + 4 (l / 32) + i % 4 in registers i = 0 .. 15.
// An operand of sixteen inner indices is eight values a lane: of row (or column) l % 32, the inner indices 8 (l / 32) + j.  Which index a place stands for is free as long as both
// operands agree: registers 0 .. 7 and 8 .. 15 of a block are each an operand of the next product as they are, whose other operand is then read in that order.  So no
// probability travels between lanes or through memory.

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
#define LDS_AT(T, p) ((__attribute__((address_space(3))) T*)(p))

constexpr float kLog2e = 1.44269504088896340736f;

// The row of a 32 x 32 block that register i of this lane holds
__device__ __forceinline__ int block_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

template <typename T> struct Operand;
template <> struct Operand<uint16_t> {
    bf16x8 v;
    static __device__ __forceinline__ Operand of(const float* p) {                  // rounded to nearest even
        u32x4 w;
        w.x = bf16_pack2(p[0], p[1]); w.y = bf16_pack2(p[2], p[3]); w.z = bf16_pack2(p[4], p[5]); w.w = bf16_pack2(p[6], p[7]);
        return {__builtin_bit_cast(bf16x8, w)};
    }
    static __device__ __forceinline__ Operand at(const void* p) { return {__builtin_bit_cast(bf16x8, *static_cast<const u32x4*>(p))}; }
    static __device__ __forceinline__ Operand zero() { return {__builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0})}; }
    __device__ __forceinline__ float operator[](int j) const {
        const u32x4 w = __builtin_bit_cast(u32x4, v);
        return j & 1 ? __uint_as_float(w[j / 2] & 0xffff0000u) : bf16_value(w[j / 2]);
    }
};
template <> struct Operand<float> {
    f32x4 lo, hi;
    static __device__ __forceinline__ Operand of(const float* p) { return {{p[0], p[1], p[2], p[3]}, {p[4], p[5], p[6], p[7]}}; }
    static __device__ __forceinline__ Operand at(const void* p) { return {static_cast<const f32x4*>(p)[0], static_cast<const f32x4*>(p)[1]}; }
    static __device__ __forceinline__ Operand zero() { return {{0, 0, 0, 0}, {0, 0, 0, 0}}; }
    __device__ __forceinline__ float operator[](int j) const { return j < 4 ? lo[j & 3] : hi[j & 3]; }
};
__device__ __forceinline__ void product(f32x16& c, const Operand<uint16_t>& a, const Operand<uint16_t>& b) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0); }
__device__ __forceinline__ void product(f32x16& c, const Operand<float>& a, const Operand<float>& b) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
}

template <typename T> __device__ __forceinline__ void put4(T* p, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
    else *reinterpret_cast<u32x2*>(p) = u32x2{bf16_pack2(a, b), bf16_pack2(c, d)};
}

// Loads into the local memory: 64 lanes' sixteen (four) bytes of a buffer, each from an offset of its own, one behind the other from `to` on; beyond the buffer's bytes zeros.  In assembly, since
// the compiler has every later read of the local memory wait for its builtin's, which leaves nothing of fetching ahead (backward pass of 2 x 4096 tokens, 32 heads of 64: 566 us, 528 so).  No register
// is written: the loads count for loads_done() alone.
__device__ __forceinline__ u32x4 buffer(const void* base, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    return {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffffu)), bytes, 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)LDS_AT(const void, p)); }
__device__ __forceinline__ void load_lds16(u32x4 from, const void* to, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_address(to)), "v"(offset), "s"(from) : "memory", "m0");
}
// the same past the caches
__device__ __forceinline__ void load_lds16_past(u32x4 from, const void* to, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds_address(to)), "v"(offset), "s"(from) : "memory", "m0");
}
__device__ __forceinline__ void load_lds4(u32x4 from, const void* to, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds_address(to)), "v"(offset), "s"(from) : "memory", "m0");
}

// ROWS rows of DP elements in the local memory: strips of 64 bytes of all rows, one strip behind the other, a row's four pieces of 16 bytes exchanged with bits 2 and 3 of its number.  Sixteen
// rows at one column then touch all banks, as four rows at 64 bytes do; and a lane's places are two numbers, whatever the strip and the sixteen rows, to which the instructions
// themselves add the rest (with whole rows behind one another, exchanged over sixteen pieces, the places took 40 registers).
template <typename T, int DP, int ROWS> struct Tile {
    static constexpr int kRowBytes = DP * (int)sizeof(T), kStrip = ROWS * 64, kBytes = ROWS * kRowBytes;
    static __device__ __forceinline__ int turn(int row) { return row >> 2 & 3; }

    // the rows from global memory by THREADS threads, without a register between: those before `low`, from `rows` on and pieces behind the row's bytes are zeros.  at(row): a row's
    // offset from base, below 2^31 - 512.  The data are there when the wavefront has waited for its loads.
    template <int THREADS, typename At> static __device__ __forceinline__ void fill(char* tile, const char* base, int low, int rows, int row_bytes, int thread, At&& at) {
        constexpr int kSlots = kBytes / 16, kEach = (kSlots + THREADS - 1) / THREADS;
        static_assert(kSlots % 64 == 0 && THREADS % 64 == 0, "whole wavefronts");
        const u32x4 from = buffer(base, 0x7fffffffu);
        const uint32_t count = rows > low ? (uint32_t)(rows - low) : 0u;     // a tile may lie behind the last row
        const int first = __builtin_amdgcn_readfirstlane(thread & ~63);
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            if (kSlots % THREADS != 0 && u * THREADS + first >= kSlots) break;     // the last pieces are fewer wavefronts'
            const int slot = u * THREADS + thread, row = slot / 4 % ROWS, piece = slot / (4 * ROWS) * 4 + ((slot & 3) ^ turn(row));
            // an offset beyond the buffer reads zeros
            const uint32_t off = (uint32_t)(row - low) < count && piece * 16 < row_bytes ? (uint32_t)(at(row) + piece * 16) : 0x80000000u;
            load_lds16(from, tile + (u * THREADS + first) * 16, off);
        }
    }

    // operand of rows row0 + l % 32 (row0 a multiple of 16): inner indices 16 step .. of the rows' elements
    static __device__ __forceinline__ Operand<T> rows(const char* tile, int row0, int step, int lane) {
        const int half = lane >> 5, at = (lane & 31) * 64, t = turn(lane & 31);
        if constexpr (sizeof(T) == 2) {
            return Operand<T>::at(tile + row0 * 64 + step / 2 * kStrip + at + (((2 * (step & 1) + half) ^ t) << 4));
        } else {
            Operand<T> o;
            o.lo = *reinterpret_cast<const f32x4*>(tile + row0 * 64 + step * kStrip + at + (((2 * half) ^ t) << 4));
            o.hi = *reinterpret_cast<const f32x4*>(tile + row0 * 64 + step * kStrip + at + (((2 * half + 1) ^ t) << 4));
            return o;
        }
    }
    // operand of columns col0 + l % 32: inner indices are the rows row0 .. row0 + 15, in the order of a block's registers
    static __device__ __forceinline__ Operand<T> columns(const char* tile, int row0, int col0, int lane) {
        const int half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // four rows of sixteen lanes' four columns each come back as a lane's column of four rows
            const int i = lane & 15, piece = (lane & 16) / 8 + (i & 3) / 2;
            const char* row = tile + row0 * 64 + col0 / 32 * kStrip + (4 * half + (i >> 2)) * 64 + (i & 1) * 8;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_AT(s16x4, row + ((piece ^ half) << 4)));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_AT(s16x4, row + 512 + ((piece ^ half ^ 2) << 4)));
            const u32x2 p = __builtin_bit_cast(u32x2, a), q = __builtin_bit_cast(u32x2, b);
            return {__builtin_bit_cast(bf16x8, (u32x4{p.x, p.y, q.x, q.y}))};
        } else {
            float v[8];
            const int i = lane & 15;
            const char* row = tile + row0 * 64 + (col0 / 16 + (lane >> 4 & 1)) * kStrip + 4 * half * 64 + (i & 3) * 4;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const float*>(row + (8 * (j / 4) + j % 4) * 64 + (((i >> 2) ^ half ^ (2 * (j / 4))) << 4));
            return Operand<T>::of(v);
        }
    }
};

// The same with whole rows behind one another, their pieces exchanged with the row's number over the row: a wavefront's load takes whole rows, not 64 bytes of each of sixteen, which counts
// where the memory is the bound (32 tokens over caches of up to 8192 keys: 94 us in strips, 85 in rows).  What is loaded is looked at once and goes past the caches (from memory, not from the
// last-level cache, 69 us and 60).
template <typename T, int DP, int ROWS> struct RowTile {
    static constexpr int kRowBytes = DP * (int)sizeof(T), kPieces = kRowBytes / 16, kBytes = ROWS * kRowBytes;
    // below kTurns, of which a row has a whole number: an exchanged piece stays in its row
    static constexpr int kTurns = sizeof(T) == 2 && kPieces == 16 ? 16 : 8;
    static_assert(kPieces % kTurns == 0, "pieces stay in their row");
    static __device__ __forceinline__ int turn(int row) {
        if constexpr (sizeof(T) == 4) return (row & 3) << 1 | (row >> 2 & 1);
        else if constexpr (kPieces == 16) return (row & 3) << 2 | (row >> 2 & 3);
        else return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    }
    static __device__ __forceinline__ int place(int row, int piece) { return row * kRowBytes + ((piece ^ turn(row)) << 4); }

    template <int THREADS, bool PAST, typename At> static __device__ __forceinline__ void fill(char* tile, const char* base, int low, int rows, int row_bytes, int thread, At&& at) {
        constexpr int kEach = kBytes / 16 / THREADS;
        static_assert(kEach * THREADS * 16 == kBytes, "whole pieces a thread");
        const u32x4 from = buffer(base, 0x7fffffffu);
        const uint32_t count = rows > low ? (uint32_t)(rows - low) : 0u;     // a tile may lie behind the last row
        const int first = __builtin_amdgcn_readfirstlane(thread & ~63);
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int slot = u * THREADS + thread, row = slot / kPieces, piece = (slot % kPieces) ^ turn(row);
            const uint32_t off = (uint32_t)(row - low) < count && piece * 16 < row_bytes ? (uint32_t)(at(row) + piece * 16) : 0x80000000u;
            if constexpr (PAST) load_lds16_past(from, tile + (u * THREADS + first) * 16, off);
            else load_lds16(from, tile + (u * THREADS + first) * 16, off);
        }
    }
    static __device__ __forceinline__ Operand<T> rows(const char* tile, int row0, int step, int lane) {
        const int row = row0 + (lane & 31), half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            return Operand<T>::at(tile + place(row, 2 * step + half));
        } else {
            Operand<T> o;
            o.lo = *reinterpret_cast<const f32x4*>(tile + place(row, 4 * step + 2 * half));
            o.hi = *reinterpret_cast<const f32x4*>(tile + place(row, 4 * step + 2 * half + 1));
            return o;
        }
    }
    static __device__ __forceinline__ Operand<T> columns(const char* tile, int row0, int col0, int lane) {
        const int half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            const int i = lane & 15, row = row0 + 4 * half + (i >> 2), col = col0 + (lane & 16) + (i & 3) * 4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_AT(s16x4, tile + place(row, col >> 3) + (col & 4) * 2));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_AT(s16x4, tile + place(row + 8, col >> 3) + (col & 4) * 2));
            const u32x2 p = __builtin_bit_cast(u32x2, a), q = __builtin_bit_cast(u32x2, b);
            return {__builtin_bit_cast(bf16x8, (u32x4{p.x, p.y, q.x, q.y}))};
        } else {
            float v[8];
            const int col = col0 + (lane & 31);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const float*>(tile + place(row0 + 8 * (j / 4) + 4 * half + j % 4, col >> 2) + (col & 3) * 4);
            return Operand<T>::of(v);
        }
    }
};

// all but the last LEFT loads that the wavefront has begun are there.  (The builtin: the compiler sees that its own loads before a loop need no wait within it.)
template <int LEFT = 0> __device__ __forceinline__ void loads_done() {
    if constexpr (LEFT == 0) {
        __builtin_amdgcn_s_waitcnt(0x0f70);
        asm volatile("" ::: "memory");
    } else {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
    }
}

// of a number that everything in a branch depends on: what few tiles need stays there.  Without it the compiler does that for all tiles and selects (a border costs a hundred vector
// instructions a tile).
template <typename V> __device__ __forceinline__ void stay_a_branch(V& v) { asm volatile("" : "+v"(v)); }

// over the two halves that share a column, for both
__device__ __forceinline__ float halves_sum(float v) {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}
__device__ __forceinline__ float halves_max(float v) {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}

// Who sees whom.  Query i stands at start + i; it sees the keys before `keys` that are not behind it (causal) and nearer than `window` (0: any).
struct Seen {
    int64_t start, window;
    int Sq, keys, causal;
    static __device__ __forceinline__ int within(int64_t v, int most) { return (int)(v < 0 ? 0 : v > most ? most : v); }
    // the keys of query i: from .. to - 1, both not falling as i grows
    __device__ __forceinline__ int from(int i) const { return window ? within(start + i - window + 1, keys) : 0; }
    __device__ __forceinline__ int to(int i) const { return causal ? within(start + i + 1, keys) : window ? within(start + i + window, keys) : keys; }
    // the queries of key j
    __device__ __forceinline__ int query_from(int j) const { return j >= keys ? Sq : causal ? within(j - start, Sq) : window ? within(j - window + 1 - start, Sq) : 0; }
    __device__ __forceinline__ int query_to(int j) const { return j >= keys ? 0 : window ? within(j + window - start, Sq) : Sq; }
};
