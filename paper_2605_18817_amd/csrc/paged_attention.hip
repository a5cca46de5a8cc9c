// Attention of new rows over a paged key-value cache.
//
//     out = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale q k_j - m),   m the largest score so far,
//
// in one pass over the visible positions j: m, sum w and sum w v are carried along and rescaled when m grows.
//
// The rows that read one key head (its G query heads times the new rows of the sequence, row r = token r / G, head r % G) go
// through the matrix cores together, 16 x RT of them in a wave, 32 positions at a time:
//     S^T = K Q^T     (16x16x32: A = 16 keys x 32 entries, B = 32 entries x 16 rows)
//     O^T += V^T P^T  (A = 16 entries x 32 keys, B = 32 keys x 16 rows)
// The result of the first product has keys 4 g + i of row r in lane 16 g + r; the second wants keys 8 g .. 8 g + 7 of row r there.  So
// the two key tiles of a step take the positions in the order that makes these the same ones (tile t, key m <-> position
// 8 (m / 4) + 4 t + m % 4), and the weights never leave their lane.  V^T is built in registers: a lane loads its 16th of the
// entries of 8 positions and exchanges 16-bit halves between them; entry e of every lane's share makes up one A operand.  Nothing
// goes through shared memory until the waves of a workgroup, which take the steps of a sequence in turn, add up.
#include "paged_rows.h"

namespace mrp {

int check_new_rows(mrp_ctx *c, const char *what, long n_rows, const mrp_new_rows *r);
int check_cache(mrp_ctx *c, const char *what, const mrp_paged_cache *k);
int check_context_device(mrp_ctx *c, const char *what);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 4;
constexpr int STEP = 32;     // positions per step of a wave

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
    constexpr uint32_t E = sizeof(T) && __is_same(T, BF16) ? 0x7f80u : 0x7c00u;
    return (v & E) == E || ((v >> 16) & E) == E;
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

// N dwords of a lane's share
template <int N>
struct Words {
    uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(const char *p) {
    Words<N> r;
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
            r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
        }
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        r.w[0] = v.x; r.w[1] = v.y;
    } else {
        r.w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
    return r;
}

template <typename T, bool E8, int HD, int RT>
__global__ __launch_bounds__(64 * WAVES) void paged_attention_kernel(const Attend A) {
    constexpr int ES = E8 ? 1 : 2;             // bytes of a cache entry
    constexpr int NC = HD / 32;                // contraction steps of a score
    constexpr int NE = HD / 16;                // entries of a lane's share of V, and A operands of O^T
    __shared__ float sm[WAVES][16 * RT], sl[WAVES][16 * RT];
    __shared__ float so[WAVES][16][HD + 4];

    const mrp_paged_cache &C = A.cache;
    const long cap = (long)C.max_pages * C.page_size;
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) check_rows(A.rows, A.n_rows, cap, A.err_flag, 64 * WAVES);
    const int b = blockIdx.z, kvh = blockIdx.y, G = A.G;
    const SeqRows s = seq_rows(A.rows, A.n_rows, cap, b);
    const int row0 = blockIdx.x * 16 * RT, nr = s.n * G;
    if (row0 >= nr) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;

    // the rows' positions and operands; lanes past the last row take it again and store nothing
    int pos[RT];
    u32x4 qf[RT][NC];
    const int t_first = row0 / G, t_last = (row0 + 16 * RT < nr ? row0 + 16 * RT - 1 : nr - 1) / G;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = row0 + 16 * rt + r16 < nr ? row0 + 16 * rt + r16 : nr - 1;
        const int t = r / G;
        pos[rt] = s.len - s.n + t;
        const uint16_t *qp = A.q + (long)(s.begin + t) * A.q_stride + (long)(kvh * G + r - t * G) * HD;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            // (8 bits: a lane's 16 bytes are 16 entries, for two contraction steps)
            const int at = E8 ? 64 * (c >> 1) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
            qf[rt][c] = *reinterpret_cast<const u32x4 *>(qp + at);
        }
    }

    // positions that any row sees: [0, sink) and [low, high); [full_low, full_high) is what all rows see
    const int p_first = s.len - s.n + t_first, p_last = s.len - s.n + t_last, W = A.attn.window;
    const bool causal = A.attn.causal != 0;
    const int high = p_last < 0 ? 0 : (causal ? p_last + 1 : s.len);
    const int full_high = p_first < 0 ? 0 : (causal ? p_first + 1 : s.len);
    const int low = W && p_first + 1 > W ? p_first + 1 - W : 0;
    const int full_low = W && p_last + 1 > W ? p_last + 1 - W : 0;
    const int sink = A.attn.n_sink;
    const int first = low / STEP;
    const int s_want = ((sink < low ? sink : low) + STEP - 1) / STEP, s_steps = s_want < first ? s_want : first;
    const int steps = high > 0 ? s_steps + (high + STEP - 1) / STEP - first : 0;

    const float c2 = A.attn.scale * 1.4426950408889634f * (E8 && C.k_scale ? C.k_scale[kvh] : 1.f);
    const long pitch = (long)C.n_kv_heads * HD * ES;      // bytes between positions
    const char *kb = static_cast<const char *>(C.k_pages) + (long)kvh * HD * ES;
    const char *vb = static_cast<const char *>(C.v_pages) + (long)kvh * HD * ES;
    const int32_t *table = A.cache.page_table + (size_t)b * C.max_pages;
    const bool whole = C.page_size % STEP == 0;           // a step lies in one page

    float m[RT], l[RT];
    f32x4 acc[RT][NE];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int e = 0; e < NE; ++e) acc[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    for (int u = wave; u < steps; u += WAVES) {
        const int key0 = (u < s_steps ? u : first + u - s_steps) * STEP;
        // places of the step's positions: one page's, or looked up by lane (key0 + lane % 32)
        int slot;
        uint32_t there = 0xffffffffu;                     // positions whose page is there
        if (whole) {
            const int page = table[key0 / C.page_size];
            if (page < 0 || page >= C.n_pages) {
                if (lane == 0) atomicOr(A.err_flag, ERR_PAGE);
                continue;
            }
            slot = page * C.page_size + key0 % C.page_size + (lane & 31);
        } else {
            const int j = key0 + (lane & 31);
            bool ok = false;
            slot = 0;
            if (j < high) {
                const int page = table[j / C.page_size];
                ok = page >= 0 && page < C.n_pages;
                if (ok) slot = page * C.page_size + j % C.page_size;
                else atomicOr(A.err_flag, ERR_PAGE);
            }
            there = (uint32_t)__ballot(ok);
        }
        const bool partial = there != 0xffffffffu || key0 + STEP > full_high || (key0 < full_low && key0 + STEP > sink);

        f32x4 sc[RT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char *kp = kb + __shfl(slot, 8 * (r16 >> 2) + 4 * t + (r16 & 3)) * pitch + 16 * g;
            u32x4 kf[NC];
            if constexpr (E8) {
#pragma unroll
                for (int c = 0; c < NC / 2; ++c) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(kp + 64 * c);
                    uint32_t a0, a1, a2, a3;
                    widen(T{}, v.x, a0, a1);
                    widen(T{}, v.y, a2, a3);
                    kf[2 * c] = u32x4{a0, a1, a2, a3};
                    widen(T{}, v.z, a0, a1);
                    widen(T{}, v.w, a2, a3);
                    kf[2 * c + 1] = u32x4{a0, a1, a2, a3};
                }
            } else {
#pragma unroll
                for (int c = 0; c < NC; ++c) kf[c] = *reinterpret_cast<const u32x4 *>(kp + 64 * c);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                sc[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NC; ++c) sc[rt][t] = mfma(T{}, kf[c], qf[rt][c], sc[rt][t]);
            }
        }
        // the lane's share of V: entries NE r16 .. of positions key0 + 8 g .. + 7
        Words<NE * ES / 4> vr[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            vr[j] = load_words<NE * ES / 4>(vb + __shfl(slot, 8 * g + j) * pitch + NE * ES * r16);
        uint32_t vw[8][NE / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (E8) {
#pragma unroll
                for (int w = 0; w < NE / 4; ++w) widen(T{}, vr[j].w[w], vw[j][2 * w], vw[j][2 * w + 1]);
            } else {
#pragma unroll
                for (int w = 0; w < NE / 2; ++w) vw[j][w] = vr[j].w[w];
            }
        }

        bool odd = false;      // values that are not finite where only some rows see them
        if (partial) {
            // scores of positions that a row does not see are dropped, values that no row sees are cleared
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const uint32_t seen = (seen_bits(pos[rt], key0, s.len, A.attn) & there) >> (8 * g);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[rt][t][i] = (seen >> (4 * t + i)) & 1u ? sc[rt][t][i] : -INFINITY;
            }
            const uint32_t any = (first_bits(high - key0) & (~first_bits(low - key0) | first_bits(sink - key0)) & there) >> (8 * g);
            bool bad = false;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < NE / 2; ++w) {
                    vw[j][w] = (any >> j) & 1u ? vw[j][w] : 0u;
                    bad |= not_finite(T{}, vw[j][w]);
                }
            odd = __any(bad);
        }

        // softmax of the step, and the weights as operands: the leading 16-bit term and the next
        u32x4 ph[RT], pl[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = m[rt];
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, fmaxf(sc[rt][0][i], sc[rt][1][i]));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float ref = mx == -INFINITY ? 0.f : mx * c2;
            if (__any(mx > m[rt])) {
                const float alpha = exp2f(m[rt] * c2 - ref);
                l[rt] *= alpha;
#pragma unroll
                for (int e = 0; e < NE; ++e) acc[rt][e] *= alpha;
            }
            m[rt] = mx;
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const float p0 = exp2f(fmaf(sc[rt][t][i], c2, -ref)), p1 = exp2f(fmaf(sc[rt][t][i + 1], c2, -ref));
                    float r0, r1, x, y;
                    sum += p0 + p1;
                    ph[rt][2 * t + i / 2] = pack2(T{}, p0, p1, r0, r1);
                    pl[rt][2 * t + i / 2] = pack2(T{}, r0, r1, x, y);
                }
            l[rt] += sum;
        }

        if (!odd) {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                u32x4 vt;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    vt[k] = __builtin_amdgcn_perm(vw[2 * k + 1][e / 2], vw[2 * k][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    acc[rt][e] = mfma(T{}, vt, ph[rt], acc[rt][e]);
                    acc[rt][e] = mfma(T{}, vt, pl[rt], acc[rt][e]);
                }
            }
        } else {
            // a weight of zero times such a value is not zero: row by row, with the values that the row sees
            for (int rr = 0; rr < 16; ++rr)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const uint32_t keep = seen_bits(__shfl(pos[rt], rr), key0, s.len, A.attn) >> (8 * g);
#pragma unroll
                    for (int e = 0; e < NE; ++e) {
                        u32x4 vt;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            vt[k] = __builtin_amdgcn_perm(vw[2 * k + 1][e / 2], vw[2 * k][e / 2], e & 1 ? 0x07060302u : 0x05040100u) &
                                    (((keep >> (2 * k)) & 1u ? 0xffffu : 0u) | ((keep >> (2 * k + 1)) & 1u ? 0xffff0000u : 0u));
                        const f32x4 d = mfma(T{}, vt, pl[rt], mfma(T{}, vt, ph[rt], f32x4{0.f, 0.f, 0.f, 0.f}));
                        if (r16 == rr) acc[rt][e] += d;
                    }
                }
        }
    }

    // the four lanes of a row add up their sums, the waves their rows
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16);
        l[rt] += __shfl_xor(l[rt], 32);
        if (g == 0) {
            sm[wave][16 * rt + r16] = m[rt];
            sl[wave][16 * rt + r16] = l[rt];
        }
    }
    const float v_scale = E8 && C.v_scale ? C.v_scale[kvh] : 1.f;
    for (int rt = 0; rt < RT; ++rt) {
        __syncthreads();
        {
            float mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, sm[w][16 * rt + r16]);
            float mine = 0.f;
            f32x4 a[NE];
#pragma unroll
            for (int q = 0; q < RT; ++q)
                if (q == rt) {
                    mine = m[q];
#pragma unroll
                    for (int e = 0; e < NE; ++e) a[e] = acc[q][e];
                }
            const float f = mine == -INFINITY ? 0.f : exp2f((mine - mx) * c2);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < NE; e += 4)
                    *reinterpret_cast<float4 *>(&so[wave][r16][NE * (4 * g + i) + e]) =
                        make_float4(a[e][i] * f, a[e + 1][i] * f, a[e + 2][i] * f, a[e + 3][i] * f);
        }
        __syncthreads();
        const int rr = threadIdx.x >> 4, part = threadIdx.x & 15, r = row0 + 16 * rt + rr;
        if (r < nr) {
            float mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, sm[w][16 * rt + rr]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                if (sm[w][16 * rt + rr] != -INFINITY) sum += sl[w][16 * rt + rr] * exp2f((sm[w][16 * rt + rr] - mx) * c2);
            const float f = mx == -INFINITY ? 0.f : v_scale / sum;
            const int t = r / G;
            const long row = s.begin + t, h = kvh * G + r - t * G;
            float o[NE];
#pragma unroll
            for (int e = 0; e < NE; ++e)
                o[e] = mx == -INFINITY ? 0.f
                                       : (((so[0][rr][NE * part + e] + so[1][rr][NE * part + e]) + so[2][rr][NE * part + e]) + so[3][rr][NE * part + e]) * f;
            uint32_t *dst = reinterpret_cast<uint32_t *>(A.out + (row * A.attn.n_heads + h) * HD + NE * part);
            float x, y;
#pragma unroll
            for (int e = 0; e < NE; e += 2) dst[e / 2] = pack2(T{}, o[e], o[e + 1], x, y);
            if (A.lse && part == 0) A.lse[row * A.attn.n_heads + h] = mx == -INFINITY ? -INFINITY : mx * c2 * 0.6931471805599453f + logf(sum);
        }
    }
}

int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

template <typename T, bool E8, int HD>
void launch(const Attend &a, hipStream_t st) {
    const long rows = (long)a.G * (a.rows.max_new < a.n_rows ? a.rows.max_new : a.n_rows);
    if (rows <= 16)
        paged_attention_kernel<T, E8, HD, 1><<<dim3(1, a.cache.n_kv_heads, a.rows.B), 64 * WAVES, 0, st>>>(a);
    else if (rows <= 32 || HD == 256)
        paged_attention_kernel<T, E8, HD, 2><<<dim3(ceil_div(rows, 32), a.cache.n_kv_heads, a.rows.B), 64 * WAVES, 0, st>>>(a);
    else if constexpr (HD < 256)
        paged_attention_kernel<T, E8, HD, 4><<<dim3(ceil_div(rows, 64), a.cache.n_kv_heads, a.rows.B), 64 * WAVES, 0, st>>>(a);
}

template <typename T, bool E8>
void launch_hd(const Attend &a, hipStream_t st) {
    if (a.cache.head_dim == 64) launch<T, E8, 64>(a, st);
    else if (a.cache.head_dim == 128) launch<T, E8, 128>(a, st);
    else launch<T, E8, 256>(a, st);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#define CHECK(expr)                       \
    do {                                  \
        const int rc_ = (expr);           \
        if (rc_ != MRP_OK) return rc_;    \
    } while (0)

}  // namespace
}  // namespace mrp

using namespace mrp;

extern "C" {

size_t mrp_paged_attention_scratch_bytes(const mrp_ctx *c, long n_rows, const mrp_new_rows *rows, const mrp_paged_cache *cache,
                                         const mrp_attn *attn) {
    (void)c; (void)n_rows; (void)rows; (void)cache; (void)attn;
    return 0;
}

int mrp_paged_attention(mrp_ctx *c, void *stream, long n_rows, const mrp_new_rows *rows, const mrp_paged_cache *cache,
                        const mrp_attn *attn, const void *q, long q_stride, void *out, float *lse, void *scratch, size_t scratch_bytes) {
    const char *what = "mrp_paged_attention";
    if (!c) return MRP_ERR_NULL;
    if (!rows || !cache || !attn) return ctx_fail(c, MRP_ERR_NULL, "%s: NULL pointer", what);
    CHECK(check_new_rows(c, what, n_rows, rows));
    CHECK(check_cache(c, what, cache));
    if (attn->n_heads < 1 || attn->n_heads > 1024 || attn->n_heads % cache->n_kv_heads)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d heads over %d key heads", what, attn->n_heads, cache->n_kv_heads);
    if (n_rows * (attn->n_heads / cache->n_kv_heads) > (1L << 26))
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %ld rows of %d heads are too many", what, n_rows, attn->n_heads);
    if ((attn->dtype != MRP_DTYPE_BF16 && attn->dtype != MRP_DTYPE_F16) || (cache->dtype != MRP_DTYPE_E4M3 && cache->dtype != attn->dtype))
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: no form for type %d over a cache of type %d", what, attn->dtype, cache->dtype);
    if (!(attn->scale > 0.f) || attn->scale > 3e38f || attn->causal < 0 || attn->causal > 1 || attn->window < 0 || attn->n_sink < 0)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: scale=%g causal=%d window=%d n_sink=%d out of range", what, (double)attn->scale, attn->causal,
                        attn->window, attn->n_sink);
    if (n_rows == 0 || rows->B == 0) return MRP_OK;
    if (!q || !out) return ctx_fail(c, MRP_ERR_NULL, "%s: a required pointer is NULL", what);
    if (q_stride < (long)attn->n_heads * cache->head_dim) return ctx_fail(c, MRP_ERR_SHAPE, "%s: rows of q overlap (stride %ld)", what, q_stride);
    if (!aligned16(q) || !aligned16(out) || q_stride % 8 || !aligned16(scratch))
        return ctx_fail(c, MRP_ERR_ALIGN, "%s: base pointers and row strides must be multiples of 16 bytes", what);
    const size_t need = mrp_paged_attention_scratch_bytes(c, n_rows, rows, cache, attn);
    if (need && !scratch) return ctx_fail(c, MRP_ERR_NULL, "%s: scratch is NULL", what);
    if (scratch_bytes < need) return ctx_fail(c, MRP_ERR_WORKSPACE, "%s: scratch holds %zu of %zu bytes", what, scratch_bytes, need);
    CHECK(check_context_device(c, what));
    const Attend a = {*rows, *cache, *attn, (int)n_rows, attn->n_heads / cache->n_kv_heads, static_cast<const uint16_t *>(q), q_stride,
                      static_cast<uint16_t *>(out), lse, ctx_view(c).err_flag};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool e8 = cache->dtype == MRP_DTYPE_E4M3;
    if (attn->dtype == MRP_DTYPE_BF16) e8 ? launch_hd<BF16, true>(a, st) : launch_hd<BF16, false>(a, st);
    else e8 ? launch_hd<F16, true>(a, st) : launch_hd<F16, false>(a, st);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MRP_OK : ctx_fail(c, MRP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // extern "C"
