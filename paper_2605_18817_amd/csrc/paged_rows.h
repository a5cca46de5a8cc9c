// Element types and the rows of a ragged batch, as the kernels around a paged cache read them.
#pragma once
#include "../../include/mrp.h"
#include "mrp_kernels.h"

namespace mrp {

struct F32 {};
struct BF16 {};
struct F16 {};

__device__ __forceinline__ void load8(const void *base, long at, F32, float (&x)[8]) {
    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(base) + at);
    const float4 a = p[0], b = p[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const void *base, long at, BF16, float (&x)[8]) {
    unpack_bf16x8(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(base) + at), x);
}
__device__ __forceinline__ void load8(const void *base, long at, F16, float (&x)[8]) {
    const f16x8 v = *reinterpret_cast<const f16x8 *>(static_cast<const uint16_t *>(base) + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
// Eight entries as they lie in memory, so that several requests are under way before the first is used
template <typename T>
struct Raw8 {
    uint4 v[__is_same(T, F32) ? 2 : 1];
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// (read once: not kept in the caches in place of what is needed again)
template <typename T>
__device__ __forceinline__ Raw8<T> raw8(const void *base, long at, T) {
    Raw8<T> r;
    const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const char *>(base) + at * (__is_same(T, F32) ? 4 : 2));
#pragma unroll
    for (int i = 0; i < (__is_same(T, F32) ? 2 : 1); ++i) {
        const u32x4 x = __builtin_nontemporal_load(p + i);
        r.v[i] = make_uint4(x[0], x[1], x[2], x[3]);
    }
    return r;
}
// Eight entries, rounded once, past the caches too: 16384 rows of 40 heads of 128, bf16, 64.9 against 72.7 us, 2048 rows 10.3 against
// 12.1; what reads them next takes as long either way
template <typename T>
__device__ __forceinline__ void store8(void *base, long at, T, const float (&x)[8]) {
    u32x4 v[__is_same(T, F32) ? 2 : 1];
    if constexpr (__is_same(T, F32)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = __float_as_uint(x[e]);
    } else if constexpr (__is_same(T, BF16)) {
        bf16x8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (__bf16)x[e];
        v[0] = __builtin_bit_cast(u32x4, h);
    } else {
        f16x8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[e];
        v[0] = __builtin_bit_cast(u32x4, h);
    }
    u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<char *>(base) + at * (__is_same(T, F32) ? 4 : 2));
#pragma unroll
    for (int i = 0; i < (__is_same(T, F32) ? 2 : 1); ++i) __builtin_nontemporal_store(v[i], p + i);
}
template <typename T>
__device__ __forceinline__ void values8(const Raw8<T> &r, float (&x)[8]) {
    if constexpr (__is_same(T, F32)) {
        x[0] = __uint_as_float(r.v[0].x); x[1] = __uint_as_float(r.v[0].y); x[2] = __uint_as_float(r.v[0].z); x[3] = __uint_as_float(r.v[0].w);
        x[4] = __uint_as_float(r.v[1].x); x[5] = __uint_as_float(r.v[1].y); x[6] = __uint_as_float(r.v[1].z); x[7] = __uint_as_float(r.v[1].w);
    } else if constexpr (__is_same(T, BF16)) {
        unpack_bf16x8(r.v[0], x);
    } else {
        const f16x8 h = __builtin_bit_cast(f16x8, r.v[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
    }
}

// Round to nearest, ties to even; beyond 448 saturates, NaN stays
__device__ __forceinline__ float e4m3_range(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }
__device__ __forceinline__ void store8_e4m3(void *base, long at, const float (&x)[8]) {
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[0]), e4m3_range(x[1]), lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[2]), e4m3_range(x[3]), lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[4]), e4m3_range(x[5]), hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[6]), e4m3_range(x[7]), hi, true);
    *reinterpret_cast<int2 *>(static_cast<uint8_t *>(base) + at) = make_int2(lo, hi);
}

// The new rows of one sequence, out of range values clamped
struct SeqRows {
    int begin, n;   // its first row, and how many
    int len;        // positions, the new rows included
};
__device__ __forceinline__ SeqRows seq_rows(const mrp_new_rows &r, int n_rows, long cap, int b) {
    SeqRows s;
    if (r.cu_rows) {
        const int a = r.cu_rows[b], e = r.cu_rows[b + 1];
        s.begin = a < 0 ? 0 : (a > n_rows ? n_rows : a);
        const int end = e > n_rows ? n_rows : e;
        s.n = end < s.begin ? 0 : end - s.begin;
    } else {
        s.begin = b * r.max_new;
        s.n = r.max_new;
    }
    if (s.n > r.max_new) s.n = r.max_new;
    const int len = r.kv_len[b];
    s.len = len < 0 ? 0 : (len > cap ? (int)cap : len);
    return s;
}
// Reports what seq_rows clamps; called by one workgroup of `threads` threads
__device__ __forceinline__ void check_rows(const mrp_new_rows &r, int n_rows, long cap, int *err_flag, int threads) {
    int bad = 0;
    for (int b = threadIdx.x; b < r.B; b += threads) {
        if (r.cu_rows) {
            const int a = r.cu_rows[b], e = r.cu_rows[b + 1];
            if (a < 0 || e < a || e > n_rows || e - a > r.max_new) bad |= ERR_ROWS;
        }
        const int len = r.kv_len[b];
        if (len < 0 || len > cap) bad |= ERR_KV_LEN;
    }
    if (bad) atomicOr(err_flag, bad);
}

}  // namespace mrp
