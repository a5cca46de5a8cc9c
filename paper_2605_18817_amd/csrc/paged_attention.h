// What the two forms of the attention over a paged cache share: element types, which positions a row sees, and how a row is stored.
#pragma once
#include "paged_rows.h"

namespace mrp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// 2^x to one unit in the last place; below 2^-126: 0
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ f32x4 mfma(BF16, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(F16, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// two values rounded to nearest, and what the rounding left
__device__ __forceinline__ uint32_t pack2(BF16, float x, float y, float &rx, float &ry) {
    const bf16x2 h = {(__bf16)x, (__bf16)y};
    rx = x - (float)h[0];
    ry = y - (float)h[1];
    return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ uint32_t pack2(F16, float x, float y, float &rx, float &ry) {
    const f16x2 h = {(_Float16)x, (_Float16)y};
    rx = x - (float)h[0];
    ry = y - (float)h[1];
    return __builtin_bit_cast(uint32_t, h);
}
// fp16 weights are carried as 2^SHIFT times themselves, through the sums as well: below 2^-14 its steps are 2^-24, whatever the weight,
// and many small weights next to a large one would drop out of the product alone.  The largest is 2^10 then (up to 32 rows of a key head, in
// two terms), or 2^7 to 2^15 where the reference may lag by 2^8; fp16 ends at 2^16.
// bf16 weights whose reference may lag are carried as 2^-8 times themselves: the sums end where those of weights of 1 would.
template <int BITS>
struct Scaled {
    static constexpr float SHIFT = BITS, ONE = BITS < 0 ? 1.f / (1 << -BITS) : 1 << BITS;
};
template <typename T>
using Few = Scaled<__is_same(T, F16) ? 10 : 0>;
template <typename T>
using Many = Scaled<__is_same(T, F16) ? 7 : -8>;
// four e4m3 values as 16-bit ones (exact in both types)
__device__ __forceinline__ void widen(BF16, uint32_t v, uint32_t &lo, uint32_t &hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.0f, true));
}
__device__ __forceinline__ void widen(F16, uint32_t v, uint32_t &lo, uint32_t &hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, true));
}
template <typename T>
__device__ __forceinline__ bool not_finite(T, uint32_t v) {   // either half
    constexpr uint32_t E = __is_same(T, BF16) ? 0x7f80u : 0x7c00u;
    return (v & E) == E || ((v >> 16) & E) == E;
}

__device__ __forceinline__ constexpr uint32_t one_bits(BF16) { return 0x3f80u; }
__device__ __forceinline__ constexpr uint32_t one_bits(F16) { return 0x3c00u; }
template <typename T>
__device__ __forceinline__ uint32_t finite_halves(T, uint32_t v) {   // halves that are not finite cleared
    constexpr uint32_t E = __is_same(T, BF16) ? 0x7f80u : 0x7c00u;
    if ((v & E) == E) v &= 0xffff0000u;
    if (((v >> 16) & E) == E) v &= 0xffffu;
    return v;
}
template <typename T>
__device__ __forceinline__ uint32_t odd_halves(T, uint32_t v) {      // 1 for halves that are not finite, else 0
    constexpr uint32_t E = __is_same(T, BF16) ? 0x7f80u : 0x7c00u;
    return ((v & E) == E ? one_bits(T{}) : 0u) | (((v >> 16) & E) == E ? one_bits(T{}) << 16 : 0u);
}

struct Attend {
    mrp_new_rows rows;
    mrp_paged_cache cache;
    mrp_attn attn;
    int n_rows, G;
    const uint16_t *q;
    long q_stride;
    uint16_t *out;
    float *lse;
    int *err_flag;
};

// bits 0 .. n - 1 of 32
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }
// which of the positions key0 .. key0 + 31 the row at position p sees
__device__ __forceinline__ uint32_t seen_bits(int p, int key0, int len, const mrp_attn &a) {
    const int high = p < 0 ? 0 : (a.causal ? p + 1 : len);
    uint32_t seen = first_bits(high - key0);
    if (a.window) seen &= ~first_bits(p + 1 - a.window - key0) | first_bits(a.n_sink - key0);
    return seen;
}

// A row's largest score starts at -inf, which is what it keeps where it sees nothing; whoever sees a position raises it to LOWEST at
// least, so that scores that are no numbers (the maximum passes them over) or -inf leave a sum of NaN or 0 and not an empty row.
constexpr float LOWEST = -3.4028234663852886e38f;
// The reference of the weights in units of log 2: finite, so that a score of -inf weighs nothing
__device__ __forceinline__ float reference(float m, float c2) { return fmaxf(m * c2, LOWEST); }

// The larger of a lane's value and that of the lane 32 (16) from it
__device__ __forceinline__ float max_halves(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float max_quarters(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// N dwords of a lane's share
template <int N>
struct Words {
    uint32_t w[N];
};
// (ONCE: past the caches, where one workgroup takes all rows of a key head.  Sequences that share pages do ask again: 64 tokens over the same
// 16384 positions 440 us, 291 through the caches, against 381 and 406 for 64 caches of their own, four rows each)
template <bool ONCE>
__device__ __forceinline__ u32x4 load_16(const char *p) {
    const u32x4 *q = reinterpret_cast<const u32x4 *>(p);
    if constexpr (ONCE) return __builtin_nontemporal_load(q);
    else return *q;
}
template <int N, bool ONCE>
__device__ __forceinline__ Words<N> load_words(const char *p) {
    Words<N> r;
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const u32x4 v = load_16<ONCE>(p + 16 * i);
            r.w[4 * i] = v[0]; r.w[4 * i + 1] = v[1]; r.w[4 * i + 2] = v[2]; r.w[4 * i + 3] = v[3];
        }
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        r.w[0] = v.x; r.w[1] = v.y;
    } else {
        r.w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
    return r;
}

// A row's part: normalised, rounded, and its log-sum (m2: the reference in units of log 2; one: the weight there)
template <typename T, int HD>
__device__ __forceinline__ void store_row(const Attend &A, long row, int head, int part, bool empty, float m2, float one, float sum, float v_scale,
                                          float (&o)[HD / 16]) {
    constexpr int NE = HD / 16;
    const float f = v_scale / sum;
    uint32_t *dst = reinterpret_cast<uint32_t *>(A.out + (row * A.attn.n_heads + head) * HD + NE * part);
    float x, y;
    Words<NE / 2> w;
#pragma unroll
    for (int e = 0; e < NE; e += 2) w.w[e / 2] = empty ? 0u : pack2(T{}, o[e] * f, o[e + 1] * f, x, y);
#pragma unroll
    for (int e = 0; e < NE / 2; ++e) dst[e] = w.w[e];
    if (A.lse && part == 0) A.lse[row * A.attn.n_heads + head] = empty ? -INFINITY : m2 * 0.6931471805599453f + logf(sum * (1.f / one));
}

// Steps of STEP positions for rows at p_first .. p_last of a sequence: [0, sink) in s_steps of them, [low, high) from step `first`
struct Steps {
    int first, s_steps, steps, low, high;
};
// Does any of these rows see position j?  (Pages of others are not looked at: behind a window they may be another sequence's, or none.)
__device__ __forceinline__ bool any_sees(const Steps &t, int n_sink, int j) { return j < t.high && (j >= t.low || j < n_sink); }
template <int STEP>
__device__ __forceinline__ Steps steps_of(const mrp_attn &a, int p_first, int p_last, int len) {
    Steps t;
    t.high = p_last < 0 ? 0 : (a.causal ? p_last + 1 : len);
    t.low = a.window && p_first + 1 > a.window ? p_first + 1 - a.window : 0;
    t.first = t.low / STEP;
    const int want = ((a.n_sink < t.low ? a.n_sink : t.low) + STEP - 1) / STEP;
    t.s_steps = want < t.first ? want : t.first;
    t.steps = t.high > 0 ? t.s_steps + (t.high + STEP - 1) / STEP - t.first : 0;
    return t;
}

// Most rows of a key head that a sequence can have
inline long most_rows(long n_rows, const mrp_new_rows &r, int G) { return (long)G * (r.max_new < n_rows ? r.max_new : n_rows); }

// Attention of many rows (prompt_attention.hip): does it take this call, its scratch, and its launch
bool prompt_takes(long rows, int head_dim);
size_t prompt_scratch_floats(long rows, int B, int n_kv_heads, long positions, int head_dim, int nCU);
hipError_t launch_prompt_attention(const Attend &a, float *scratch, int nCU, hipStream_t st);

}  // namespace mrp
