// Included inside the unnamed namespaces of attention.hip and attention_back.hip: their arguments, and what the host checks of both.

// Strides are in bytes.  R query heads share a key head; the queries of one key head's are numbered i * R + r, head r of them of query i, and called columns.
struct Heads { int64_t batch; int token, head; };
struct AttentionArgs {
    const char *q, *k, *v;
    Heads qs, ks, vs;
    const int *lengths, *starts;
    char* out;
    float *lse, *parts, *values;                        // parts of the keys: [split][group][column] their lse, and behind them on 16 bytes their values of D elements each
    int64_t window;
    int Sq, Sk, H, G, R, D, causal, groups;             // groups: B * G
    int blocks, splits, tiles;                          // of columns; parts of the keys, and how many tiles one has at least
    float scale;
};
__device__ __forceinline__ int64_t row_offset(const Heads& s, int64_t token, int head) { return token * s.token + (int64_t)head * s.head; }
template <typename A> __device__ __forceinline__ Seen seen_of(const A& a, int b) {
    Seen s;
    int n = a.Sk;
    if (a.lengths) { n = a.lengths[b]; n = n < 0 ? 0 : n > a.Sk ? a.Sk : n; }
    s.keys = n;
    s.start = a.starts ? a.starts[b] : (int64_t)a.Sk - a.Sq;
    s.window = a.window;
    s.causal = a.causal;
    s.Sq = a.Sq;
    // keys that stand behind every query's are as ones behind the sequence: a cache may hold anything there
    const int64_t behind = s.start + a.Sq;
    if (a.causal) s.keys = Seen::within(behind, s.keys);
    else if (a.window) s.keys = Seen::within(behind + a.window - 1, s.keys);
    return s;
}

// ------------------------------------------------------------------ host side

#include "launch.h"

// A tensor of rows: nothing behind what 31 bits say of a tile's rows, which are up to 129 tokens' of the `share` heads that have one key head; every row on 16 bytes
constexpr int64_t kMostStride = 1 << 23, kMostHeads = 1 << 30, kMostTokens = 1 << 29, kMostGroups = 1 << 24;
int check_heads(const void* p, const int64_t* strides, int64_t B, int64_t share, int64_t es) {
    const int64_t per = 16 / es;
    if (strides[0] < 0 || strides[1] < 0 || strides[2] < 0) return DIVISION_EINVAL;
    if (!aligned(p, 16) || strides[0] % per || strides[1] % per || strides[2] % per) return DIVISION_EALIGN;
    if (strides[1] > kMostStride / es || strides[2] > kMostHeads / es / share || strides[0] > (int64_t(1) << 40) / B) return DIVISION_ERANGE;
    return DIVISION_OK;
}
int check_attention(const division_attention& a) {
    if (!type_ok(a.dt)) return DIVISION_EINVAL;
    if (a.B < 0 || a.Sq < 0 || a.Sk < 0 || a.H < 1 || a.G < 1 || a.H % a.G || a.D < 8 || a.D > 128 || a.D % 8 || a.window < 0 || (a.causal != 0 && a.causal != 1)) return DIVISION_EINVAL;
    if (!(a.scale > 0.0f && a.scale <= 2e38f)) return DIVISION_EINVAL;
    if (!aligned(a.lengths, 4) || !aligned(a.starts, 4)) return DIVISION_EALIGN;
    if (a.B == 0) return DIVISION_OK;
    const int64_t es = (int64_t)size_of(a.dt), R = a.H / a.G;
    if (a.B > (1 << 24) || a.H > 4096 || a.Sq > kMostTokens || a.Sk > kMostTokens || a.Sq * R > (int64_t(1) << 30)) return DIVISION_ERANGE;
    // more than any launch has room for, before it is narrowed
    if ((a.Sq > 0 || a.Sk > 0) && a.B * a.G >= kMostGroups) return DIVISION_ERANGE;
    if (a.Sq > 0) CHECKED(check_heads(a.q, a.q_strides, a.B, R, es));
    if (a.Sk > 0) {
        CHECKED(check_heads(a.k, a.k_strides, a.B, 1, es));
        CHECKED(check_heads(a.v, a.v_strides, a.B, 1, es));
    }
    return DIVISION_OK;
}
Heads heads_of(const int64_t* strides, int64_t es) { return {strides[0] * es, (int)(strides[1] * es), (int)(strides[2] * es)}; }
AttentionArgs args_of(const division_attention& a) {
    const int64_t es = (int64_t)size_of(a.dt);
    AttentionArgs r{};
    r.q = static_cast<const char*>(a.q); r.k = static_cast<const char*>(a.k); r.v = static_cast<const char*>(a.v);
    r.qs = heads_of(a.q_strides, es); r.ks = heads_of(a.k_strides, es); r.vs = heads_of(a.v_strides, es);
    r.lengths = a.lengths; r.starts = a.starts;
    // beyond all positions a window of any size is the same
    r.window = a.window > (int64_t(1) << 40) ? (int64_t(1) << 40) : a.window;
    r.Sq = (int)a.Sq; r.Sk = (int)a.Sk; r.H = (int)a.H; r.G = (int)a.G; r.R = (int)(a.H / a.G); r.D = (int)a.D;
    r.causal = a.causal; r.groups = (int)(a.B * a.G); r.scale = a.scale;
    return r;
}
