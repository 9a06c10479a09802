// Included inside the unnamed namespaces of masks.hip and dropout_add.hip: which elements dropout keeps, with a stored mask and without.

constexpr uint32_t kWeyl = 0x9E3779B9u;
constexpr uint64_t kDropoutStream = 0xD509A5B3C2E1F047ull;

// 32-bit xorshift-multiply finaliser (shifts 16/15/16): the codec's random source
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16; x *= 0x7feb352du;
    x ^= x >> 15; x *= 0x846ca68bu;
    x ^= x >> 16;
    return x;
}

// random word of element pair j of a stream segment with keys (k1, k2)
__device__ __forceinline__ uint32_t pair_word(uint32_t k1, uint32_t k2, uint32_t j) {
    uint32_t x = k1 + j * kWeyl;
    x ^= x >> 16; x *= 0x7feb352du;
    x = __builtin_amdgcn_bitop3_b32(x, x >> 15, k2, 0x96); x *= 0x846ca68bu;      // exclusive or of the three, which the compiler does not always make one instruction of
    x ^= x >> 16;
    return x;
}
