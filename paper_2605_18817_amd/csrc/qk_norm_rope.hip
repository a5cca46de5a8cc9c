// Norm and rotation of the heads of q and k, their gradient, and the same on the way into a paged cache.
//
//     n = x / sqrt(mean(x^2) + eps) * gain,   y = R(p) n      (R turns the pairs (j, j + r), j < r = rotary_dim / 2)
//
// The gradient turns back, dn = R(p)^T dy (R is orthogonal), and with i = 1 / sqrt(mean(x^2) + eps) and t = dn * gain:
//     dgain = sum over rows and heads of dn x i,      dx = i t - x i^3 mean(x t).
//
// head_dim / 16 threads share a head and each holds 16 of its entries, as two chunks of 8 that hold both members of their
// pairs: the rotation needs no exchange between threads, the norm a sum over 4, 8 or 16 neighbours.  All arithmetic is in
// 32 bits; every output is rounded once.  The kernels move each input and output once and compute next to nothing: 16384 rows of 32 +
// 8 heads of 128, bf16, forward 64 us (338 MB, 5.25 TB/s), gradient 115 (505 MB, 4.4); 13 thousand rows appended, fp16, 64 us (307 MB).
#include "paged_rows.h"

namespace mrp {

namespace {

// The thread's two chunks of a head: the first entries of each
__device__ __forceinline__ void chunk_places(int c, int rot, int &o0, int &o1) {
    if (c < rot / 16) {
        o0 = 8 * c;
        o1 = rot / 2 + 8 * c;
    } else {
        o0 = rot + 16 * (c - rot / 16);
        o1 = o0 + 8;
    }
}

__device__ __forceinline__ void load_gain(const void *gain, int dtype, int at, float (&g)[8]) {
    if (dtype == MRP_DTYPE_F32) load8(gain, at, F32{}, g);
    else if (dtype == MRP_DTYPE_BF16) load8(gain, at, BF16{}, g);
    else load8(gain, at, F16{}, g);
}

// Sum over the `tph` threads of a head
__device__ __forceinline__ float head_sum(float x, int tph) {
    for (int off = 1; off < tph; off <<= 1) x += __shfl_xor(x, off);
    return x;
}

__device__ __forceinline__ float sum_squares(const float (&a)[8], const float (&b)[8]) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += a[e] * a[e] + b[e] * b[e];
    return s;
}

struct Turn {
    float c[8], s[8];
};
__device__ __forceinline__ Turn load_turn(const mrp_qk &qk, int pos, int c) {
    Turn t;
    const float4 *p = reinterpret_cast<const float4 *>(qk.rope + ((size_t)pos * (qk.rotary_dim / 2) + 8 * c) * 2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float4 v = p[e];
        t.c[2 * e] = v.x; t.s[2 * e] = v.y; t.c[2 * e + 1] = v.z; t.s[2 * e + 1] = v.w;
    }
    return t;
}

__device__ __forceinline__ int clamp_pos(int pos, int n_pos, int *err_flag) {
    if (pos >= 0 && pos < n_pos) return pos;
    atomicOr(err_flag, ERR_POSITION);
    return pos < 0 ? 0 : n_pos - 1;
}

// a, b <- the head's normalised, scaled and rotated chunks
__device__ __forceinline__ void norm_turn(const mrp_qk &qk, const void *gain, int pos, int c, int o0, int o1, int tph,
                                          int *err_flag, float (&a)[8], float (&b)[8]) {
    if (gain) {
        float g0[8], g1[8];
        load_gain(gain, qk.gain_dtype, o0, g0);
        load_gain(gain, qk.gain_dtype, o1, g1);
        const float ss = head_sum(sum_squares(a, b), tph);
        const float inv = 1.0f / sqrtf(ss / (float)qk.head_dim + qk.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a[e] = a[e] * inv * g0[e];
            b[e] = b[e] * inv * g1[e];
        }
    }
    if (c < qk.rotary_dim / 16) {
        const Turn t = load_turn(qk, clamp_pos(pos, qk.n_pos, err_flag), c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = a[e], y = b[e];
            a[e] = x * t.c[e] - y * t.s[e];
            b[e] = y * t.c[e] + x * t.s[e];
        }
    }
}

struct QkForward {
    mrp_qk qk;
    long n_rows;
    const int32_t *pos;
    const void *q, *k;
    long q_stride, k_stride;
    void *q_out, *k_out;
    int *err_flag;
};

template <typename XT, typename YT>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const QkForward A) {
    const mrp_qk &qk = A.qk;
    const int tph = qk.head_dim / 16, c = threadIdx.x & (tph - 1);
    const int heads = qk.n_heads + qk.n_kv_heads;
    const long item = ((long)blockIdx.x * 256 + threadIdx.x) / tph;
    const long row = item / heads;
    const int h = (int)(item - row * heads);
    if (row >= A.n_rows) return;   // (all threads of a head)
    int o0, o1;
    chunk_places(c, qk.rotary_dim, o0, o1);
    const bool is_q = h < qk.n_heads;
    const int hh = is_q ? h : h - qk.n_heads;
    const void *src = is_q ? A.q : A.k;
    const long at = row * (is_q ? A.q_stride : A.k_stride) + (long)hh * qk.head_dim;
    float a[8], b[8];
    values8(raw8(src, at + o0, XT{}), a);
    values8(raw8(src, at + o1, XT{}), b);
    norm_turn(qk, is_q ? qk.q_gain : qk.k_gain, qk.rotary_dim ? A.pos[row] : 0, c, o0, o1, tph, A.err_flag, a, b);
    void *dst = is_q ? A.q_out : A.k_out;
    const long to = (row * (is_q ? qk.n_heads : qk.n_kv_heads) + hh) * qk.head_dim;
    store8(dst, to + o0, YT{}, a);
    store8(dst, to + o1, YT{}, b);
}

struct QkGrad {
    QkForward f;               // q_out, k_out: the gradients of the outputs (read)
    void *dq, *dk;
    long dq_stride, dk_stride;
    int wg_q, wg_k;            // workgroups on q and on k
    float *part;               // [wg_q + wg_k][head_dim]
    float *dq_gain, *dk_gain;
};

template <typename XT, typename YT>
__global__ __launch_bounds__(256) void qk_norm_rope_grad_kernel(const QkGrad A) {
    __shared__ float sums[256][16];
    const mrp_qk &qk = A.f.qk;
    const int tph = qk.head_dim / 16, c = threadIdx.x & (tph - 1), per = 256 / tph;
    const bool is_q = (int)blockIdx.x < A.wg_q;
    const int w = is_q ? blockIdx.x : blockIdx.x - A.wg_q, nw = is_q ? A.wg_q : A.wg_k;
    const int heads = is_q ? qk.n_heads : qk.n_kv_heads;
    const void *x = is_q ? A.f.q : A.f.k, *dy = is_q ? A.f.q_out : A.f.k_out, *gain = is_q ? qk.q_gain : qk.k_gain;
    void *dx = is_q ? A.dq : A.dk;
    const long stride = is_q ? A.f.q_stride : A.f.k_stride, dstride = is_q ? A.dq_stride : A.dk_stride;
    int o0, o1;
    chunk_places(c, qk.rotary_dim, o0, o1);
    float g0[8], g1[8], s0[8], s1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s0[e] = s1[e] = 0.f;
    if (gain) {
        load_gain(gain, qk.gain_dtype, o0, g0);
        load_gain(gain, qk.gain_dtype, o1, g1);
    }
    const long items = A.f.n_rows * heads, step = (long)nw * per;
    // two heads at a time: all that they read is asked for before the first is worked on
    for (long item = (long)w * per + threadIdx.x / tph; item < items; item += 2 * step) {
        Raw8<YT> y0[2], y1[2];
        Raw8<XT> x0[2], x1[2];
        long at[2];
        int pos[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const long it = item + u * step < items ? item + u * step : item, row = it / heads;
            at[u] = (it - row * heads) * qk.head_dim;
            pos[u] = qk.rotary_dim ? A.f.pos[row] : 0;
            y0[u] = raw8(dy, it * qk.head_dim + o0, YT{});
            y1[u] = raw8(dy, it * qk.head_dim + o1, YT{});
            if (gain) {
                x0[u] = raw8(x, row * stride + at[u] + o0, XT{});
                x1[u] = raw8(x, row * stride + at[u] + o1, XT{});
            }
            at[u] += row * dstride;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (item + u * step >= items) break;   // (all threads of a head)
            float a[8], b[8], t0[8], t1[8];
            values8(y0[u], t0);
            values8(y1[u], t1);
            if (c < qk.rotary_dim / 16) {          // dn = R^T dy
                const Turn t = load_turn(qk, clamp_pos(pos[u], qk.n_pos, A.f.err_flag), c);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = t0[e], q = t1[e];
                    t0[e] = p * t.c[e] + q * t.s[e];
                    t1[e] = q * t.c[e] - p * t.s[e];
                }
            }
            if (gain) {
                values8(x0[u], a);
                values8(x1[u], b);
                const float inv = 1.0f / sqrtf(head_sum(sum_squares(a, b), tph) / (float)qk.head_dim + qk.eps);
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s0[e] += t0[e] * a[e] * inv;
                    s1[e] += t1[e] * b[e] * inv;
                    t0[e] *= g0[e];
                    t1[e] *= g1[e];
                    dot += t0[e] * a[e] + t1[e] * b[e];
                }
                const float m = head_sum(dot, tph) / (float)qk.head_dim * inv * inv;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t0[e] = inv * (t0[e] - a[e] * m);
                    t1[e] = inv * (t1[e] - b[e] * m);
                }
            }
            store8(dx, at[u] + o0, XT{}, t0);
            store8(dx, at[u] + o1, XT{}, t1);
        }
    }
    if (!gain || !(is_q ? A.dq_gain : A.dk_gain)) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sums[threadIdx.x][e] = s0[e];
        sums[threadIdx.x][8 + e] = s1[e];
    }
    __syncthreads();
    // entry j of the head: which thread of a head and which of its 16 sums
    for (int j = threadIdx.x; j < 16 * tph; j += 256) {
        const int cc = j >> 4, e = j & 15;
        float s = 0.f;
        for (int u = 0; u < per; ++u) s += sums[u * tph + cc][e];
        int p0, p1;
        chunk_places(cc, qk.rotary_dim, p0, p1);
        A.part[(size_t)blockIdx.x * qk.head_dim + (e < 8 ? p0 + e : p1 + e - 8)] = s;
    }
}

// The workgroups' sums: 64 threads on an entry take every 64th, then a tree over them (the order is the same in every call)
__global__ __launch_bounds__(1024) void gain_sum_kernel(const QkGrad A) {
    __shared__ float sums[64][17];
    const int hd = A.f.qk.head_dim, groups = hd / 16;
    const bool is_q = (int)blockIdx.x < groups;
    const int col = (is_q ? blockIdx.x : blockIdx.x - groups) * 16 + (threadIdx.x & 15), u = threadIdx.x >> 4;
    float *out = is_q ? A.dq_gain : A.dk_gain;
    if (!out || !(is_q ? A.f.qk.q_gain : A.f.qk.k_gain)) return;
    const float *part = A.part + (is_q ? 0 : (size_t)A.wg_q * hd) + col;
    const int n = is_q ? A.wg_q : A.wg_k;
    float s = 0.f;
#pragma unroll 4
    for (int w = u; w < n; w += 64) s += part[(size_t)w * hd];
    sums[u][threadIdx.x & 15] = s;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (u < half) sums[u][threadIdx.x & 15] += sums[u + half][threadIdx.x & 15];
        __syncthreads();
    }
    if (u == 0) out[col] = sums[0][threadIdx.x & 15];
}

struct Append {
    mrp_qk qk;
    mrp_new_rows rows;
    mrp_paged_cache cache;
    int n_rows;
    const void *q, *k, *v;
    long q_stride, k_stride, v_stride;
    void *q_out;
    int *err_flag;
};

template <typename XT, typename YT>
__global__ __launch_bounds__(256) void cache_append_kernel(const Append A) {
    const mrp_qk &qk = A.qk;
    const mrp_paged_cache &C = A.cache;
    const int tph = qk.head_dim / 16, c = threadIdx.x & (tph - 1);
    const int nq = A.q ? qk.n_heads : 0, nkv = C.n_kv_heads, heads = nq + 2 * nkv;
    const long cap = (long)C.max_pages * C.page_size;
    if (blockIdx.x == 0) check_rows(A.rows, A.n_rows, cap, A.err_flag, 256);
    const long item = ((long)blockIdx.x * 256 + threadIdx.x) / tph;
    const long row = item / heads;
    const int h = (int)(item - row * heads);
    if (row >= A.n_rows) return;
    // what the thread takes of its head is on its way while the row is looked up
    int o0, o1;
    chunk_places(c, qk.rotary_dim, o0, o1);
    const bool is_q = h < nq, is_k = h < nq + nkv;
    const int hh = is_q ? h : (is_k ? h - nq : h - nq - nkv);
    const void *src = is_q ? A.q : (is_k ? A.k : A.v);
    const long from = row * (is_q ? A.q_stride : (is_k ? A.k_stride : A.v_stride)) + (long)hh * qk.head_dim;
    const Raw8<XT> r0 = raw8(src, from + o0, XT{}), r1 = raw8(src, from + o1, XT{});
    // the row's sequence: the last one that begins at or before it
    int b;
    if (A.rows.cu_rows) {
        int lo = 0, hi = A.rows.B;   // first b with cu_rows[b + 1] > row
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (A.rows.cu_rows[mid + 1] > row) hi = mid;
            else lo = mid + 1;
        }
        b = lo;
    } else {
        b = (int)(row / A.rows.max_new);
    }
    if (b >= A.rows.B) return;
    const SeqRows s = seq_rows(A.rows, A.n_rows, cap, b);
    const int i = (int)row - s.begin;
    if (i < 0 || i >= s.n) return;
    const int pos = s.len - s.n + i;
    float x0[8], x1[8];
    values8(r0, x0);
    values8(r1, x1);
    if (is_q) {
        const long to = (row * nq + h) * qk.head_dim;
        if (pos < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x0[e] = x1[e] = 0.f;
        } else {
            norm_turn(qk, qk.q_gain, pos, c, o0, o1, tph, A.err_flag, x0, x1);
        }
        store8(A.q_out, to + o0, YT{}, x0);
        store8(A.q_out, to + o1, YT{}, x1);
        return;
    }
    if (pos < 0) return;
    const int page = C.page_table[(size_t)b * C.max_pages + pos / C.page_size];
    if (page < 0 || page >= C.n_pages) {
        if (c == 0) atomicOr(A.err_flag, ERR_PAGE);
        return;
    }
    if (is_k) norm_turn(qk, qk.k_gain, pos, c, o0, o1, tph, A.err_flag, x0, x1);
    const long slot = (long)page * C.page_size + pos % C.page_size;
    const long to = (slot * nkv + hh) * qk.head_dim;
    void *dst = is_k ? C.k_pages : C.v_pages;
    if (C.dtype == MRP_DTYPE_E4M3) {
        const float *scale = is_k ? C.k_scale : C.v_scale;
        const float sc = scale ? scale[hh] : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x0[e] /= sc;
            x1[e] /= sc;
        }
        store8_e4m3(dst, to + o0, x0);
        store8_e4m3(dst, to + o1, x1);
    } else if (C.dtype == MRP_DTYPE_BF16) {
        store8(dst, to + o0, BF16{}, x0);
        store8(dst, to + o1, BF16{}, x1);
    } else {
        store8(dst, to + o0, F16{}, x0);
        store8(dst, to + o1, F16{}, x1);
    }
}

__global__ __launch_bounds__(256) void rope_table_kernel(int n_pos, int half, double theta, float2 *out) {
    const long idx = (long)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (long)n_pos * half) return;
    const int j = (int)(idx % half);
    const double ang = (double)(idx / half) * pow(theta, -(double)j / (double)half);
    out[idx] = make_float2((float)cos(ang), (float)sin(ang));
}

// ---- host side

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int size_of(int dtype) { return dtype == MRP_DTYPE_F32 ? 4 : (dtype == MRP_DTYPE_E4M3 ? 1 : 2); }

// f(XT, YT) for the pair of types; false: not a pair that there is
template <typename Fn>
bool for_types(int x, int y, Fn f) {
    if (x == MRP_DTYPE_F32 && y == MRP_DTYPE_F32) f(F32{}, F32{});
    else if (x == MRP_DTYPE_F32 && y == MRP_DTYPE_BF16) f(F32{}, BF16{});
    else if (x == MRP_DTYPE_F32 && y == MRP_DTYPE_F16) f(F32{}, F16{});
    else if (x == MRP_DTYPE_BF16 && y == MRP_DTYPE_BF16) f(BF16{}, BF16{});
    else if (x == MRP_DTYPE_F16 && y == MRP_DTYPE_F16) f(F16{}, F16{});
    else return false;
    return true;
}

constexpr long MAX_ROWS = 1L << 24;
constexpr long MAX_POSITIONS = (1L << 31) - 4096;   // of a sequence: tiles are looked up ahead of the last one, with positions in an int
constexpr long MAX_THREADS = 0xffffff00L;   // of one launch

// What all calls on a mrp_qk check; the heads that are given are checked by their callers
int check_qk(mrp_ctx *c, const char *what, long n_rows, const mrp_qk *qk) {
    if (n_rows < 0 || n_rows > MAX_ROWS) return ctx_fail(c, MRP_ERR_SHAPE, "%s: n_rows=%ld out of range", what, n_rows);
    if (qk->head_dim != 64 && qk->head_dim != 128 && qk->head_dim != 256)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: head_dim %d is none of 64, 128, 256", what, qk->head_dim);
    if (qk->n_heads < 1 || qk->n_heads > 1024 || qk->n_kv_heads < 0 || qk->n_kv_heads > 1024)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d heads, %d key heads out of range", what, qk->n_heads, qk->n_kv_heads);
    if (n_rows * (qk->n_heads + 2 * qk->n_kv_heads) * (qk->head_dim / 16) > MAX_THREADS)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %ld rows of %d heads are too many", what, n_rows, qk->n_heads + 2 * qk->n_kv_heads);
    if (qk->rotary_dim < 0 || qk->rotary_dim > qk->head_dim || qk->rotary_dim % 16)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: rotary_dim %d is not a multiple of 16 in [0, head_dim]", what, qk->rotary_dim);
    if (qk->rotary_dim && (!qk->rope || qk->n_pos < 1))
        return ctx_fail(c, qk->rope ? MRP_ERR_SHAPE : MRP_ERR_NULL, "%s: rotation without a table of positions", what);
    if (!for_types(qk->x_dtype, qk->y_dtype, [](auto, auto) {}))
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: no form for types %d -> %d", what, qk->x_dtype, qk->y_dtype);
    if (qk->gain_dtype != MRP_DTYPE_F32 && qk->gain_dtype != MRP_DTYPE_BF16 && qk->gain_dtype != MRP_DTYPE_F16)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: gain type %d", what, qk->gain_dtype);
    if (!(qk->eps >= 0.f)) return ctx_fail(c, MRP_ERR_SHAPE, "%s: eps is negative", what);
    if ((qk->q_gain && !aligned16(qk->q_gain)) || (qk->k_gain && !aligned16(qk->k_gain)) || (qk->rope && !aligned16(qk->rope)))
        return ctx_fail(c, MRP_ERR_ALIGN, "%s: gains and table must be 16-byte aligned", what);
    return MRP_OK;
}

// A row tensor of `heads` heads: base pointer and stride
int check_rows_of(mrp_ctx *c, const char *what, const void *p, long stride, int heads, int head_dim, int dtype) {
    if (!p) return ctx_fail(c, MRP_ERR_NULL, "%s: a required pointer is NULL", what);
    if (stride < (long)heads * head_dim) return ctx_fail(c, MRP_ERR_SHAPE, "%s: rows of %d heads overlap (stride %ld)", what, heads, stride);
    if (!aligned16(p) || stride * size_of(dtype) % 16)
        return ctx_fail(c, MRP_ERR_ALIGN, "%s: base pointers and row strides must be multiples of 16 bytes", what);
    return MRP_OK;
}

int check_device(mrp_ctx *c, const char *what) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != ctx_view(c).device)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: the context is device %d's, the current device is %d", what, ctx_view(c).device, dev);
    return MRP_OK;
}

#define CHECK(expr)                       \
    do {                                  \
        const int rc_ = (expr);           \
        if (rc_ != MRP_OK) return rc_;    \
    } while (0)

int launched(mrp_ctx *c, const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MRP_OK : ctx_fail(c, MRP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Workgroups of the gradient on the heads of q or of k, each with sums of its own: 1024 in all, shared out by the heads (four
// on a compute unit; more are only more sums to add up)
int grad_workgroups(long n_rows, int heads, int all_heads, int head_dim) {
    const long per = 256 / (head_dim / 16), n = (n_rows * heads + per - 1) / per;
    const long most = (1024L * heads + all_heads - 1) / all_heads;
    return (int)(n > most ? most : n);
}

}  // namespace

int check_new_rows(mrp_ctx *c, const char *what, long n_rows, const mrp_new_rows *r) {
    if (n_rows < 0 || n_rows > MAX_ROWS) return ctx_fail(c, MRP_ERR_SHAPE, "%s: n_rows=%ld out of range", what, n_rows);
    if (r->B < 0 || r->B > 65535 || r->max_new < 1) return ctx_fail(c, MRP_ERR_SHAPE, "%s: B=%d max_new=%d out of range", what, r->B, r->max_new);
    if (r->B > 0 && !r->kv_len) return ctx_fail(c, MRP_ERR_NULL, "%s: kv_len is NULL", what);
    if (!r->cu_rows && (long)r->B * r->max_new > n_rows)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d sequences of %d rows, but %ld rows", what, r->B, r->max_new, n_rows);
    return MRP_OK;
}

int check_cache(mrp_ctx *c, const char *what, const mrp_paged_cache *k, int B) {
    if (!k->k_pages || !k->v_pages || (B > 0 && !k->page_table)) return ctx_fail(c, MRP_ERR_NULL, "%s: the cache has a NULL pointer", what);
    if (k->dtype != MRP_DTYPE_BF16 && k->dtype != MRP_DTYPE_F16 && k->dtype != MRP_DTYPE_E4M3)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: cache type %d", what, k->dtype);
    if (k->head_dim != 64 && k->head_dim != 128 && k->head_dim != 256)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: head_dim %d is none of 64, 128, 256", what, k->head_dim);
    if (k->n_kv_heads < 1 || k->n_kv_heads > 1024 || k->n_pages < 1 || k->page_size < 1 || k->max_pages < 1 ||
        (long)k->n_pages * k->page_size > 0x7fffffffL || (long)k->max_pages * k->page_size > MAX_POSITIONS)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d kv heads, %d pages of %d, %d a sequence out of range", what, k->n_kv_heads,
                        k->n_pages, k->page_size, k->max_pages);
    if (!aligned16(k->k_pages) || !aligned16(k->v_pages)) return ctx_fail(c, MRP_ERR_ALIGN, "%s: pages must be 16-byte aligned", what);
    if ((k->k_scale || k->v_scale) && k->dtype != MRP_DTYPE_E4M3)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: scales are for caches of E4M3", what);
    return MRP_OK;
}

int check_context_device(mrp_ctx *c, const char *what) { return check_device(c, what); }

}  // namespace mrp

using namespace mrp;

extern "C" {

int mrp_rope_table(mrp_ctx *c, void *stream, int n_pos, int rotary_dim, float theta, float *out) {
    if (!c) return MRP_ERR_NULL;
    if (!out) return ctx_fail(c, MRP_ERR_NULL, "mrp_rope_table: NULL pointer");
    if (n_pos < 1 || n_pos > (1 << 24) || rotary_dim < 16 || rotary_dim > 256 || rotary_dim % 16 || !(theta > 1.f) || theta > 3e38f)
        return ctx_fail(c, MRP_ERR_SHAPE, "mrp_rope_table: n_pos=%d rotary_dim=%d theta=%g out of range", n_pos, rotary_dim, (double)theta);
    if (!aligned16(out)) return ctx_fail(c, MRP_ERR_ALIGN, "mrp_rope_table: the table must be 16-byte aligned");
    CHECK(check_device(c, "mrp_rope_table"));
    const long n = (long)n_pos * (rotary_dim / 2);
    rope_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(n_pos, rotary_dim / 2, (double)theta,
                                                                                               reinterpret_cast<float2 *>(out));
    return launched(c, "mrp_rope_table");
}

int mrp_qk_norm_rope(mrp_ctx *c, void *stream, long n_rows, const mrp_qk *qk, const int32_t *pos, const void *q, long q_stride,
                     const void *k, long k_stride, void *q_out, void *k_out) {
    const char *what = "mrp_qk_norm_rope";
    if (!c) return MRP_ERR_NULL;
    if (!qk) return ctx_fail(c, MRP_ERR_NULL, "%s: NULL pointer", what);
    CHECK(check_qk(c, what, n_rows, qk));
    if (n_rows == 0) return MRP_OK;
    if (qk->rotary_dim && !pos) return ctx_fail(c, MRP_ERR_NULL, "%s: pos is NULL", what);
    CHECK(check_rows_of(c, what, q, q_stride, qk->n_heads, qk->head_dim, qk->x_dtype));
    CHECK(check_rows_of(c, what, q_out, (long)qk->n_heads * qk->head_dim, qk->n_heads, qk->head_dim, qk->y_dtype));
    if (qk->n_kv_heads) {
        CHECK(check_rows_of(c, what, k, k_stride, qk->n_kv_heads, qk->head_dim, qk->x_dtype));
        CHECK(check_rows_of(c, what, k_out, (long)qk->n_kv_heads * qk->head_dim, qk->n_kv_heads, qk->head_dim, qk->y_dtype));
    }
    CHECK(check_device(c, what));
    const QkForward a = {*qk, n_rows, pos, q, k, q_stride, k_stride, q_out, k_out, ctx_view(c).err_flag};
    const long threads = n_rows * (qk->n_heads + qk->n_kv_heads) * (qk->head_dim / 16);
    for_types(qk->x_dtype, qk->y_dtype, [&](auto xt, auto yt) {
        qk_norm_rope_kernel<decltype(xt), decltype(yt)><<<(unsigned)((threads + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(a);
    });
    return launched(c, what);
}

size_t mrp_qk_norm_rope_grad_scratch_bytes(long n_rows, const mrp_qk *qk) {
    if (!qk || n_rows <= 0 || n_rows > MAX_ROWS || qk->head_dim < 16 || qk->head_dim > 256 || qk->n_heads < 1 || qk->n_kv_heads < 0) return 0;
    const int all = qk->n_heads + qk->n_kv_heads;
    return (size_t)(grad_workgroups(n_rows, qk->n_heads, all, qk->head_dim) + grad_workgroups(n_rows, qk->n_kv_heads, all, qk->head_dim)) *
           qk->head_dim * sizeof(float);
}

int mrp_qk_norm_rope_grad(mrp_ctx *c, void *stream, long n_rows, const mrp_qk *qk, const int32_t *pos, const void *q, long q_stride,
                          const void *k, long k_stride, const void *dq_out, const void *dk_out, void *dq, long dq_stride, void *dk,
                          long dk_stride, float *dq_gain, float *dk_gain, void *scratch, size_t scratch_bytes) {
    const char *what = "mrp_qk_norm_rope_grad";
    if (!c) return MRP_ERR_NULL;
    if (!qk) return ctx_fail(c, MRP_ERR_NULL, "%s: NULL pointer", what);
    CHECK(check_qk(c, what, n_rows, qk));
    if ((dq_gain && !qk->q_gain) || (dk_gain && (!qk->k_gain || !qk->n_kv_heads)))
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: the gradient of a gain that there is not", what);
    if (n_rows > 0) {
        if (qk->rotary_dim && !pos) return ctx_fail(c, MRP_ERR_NULL, "%s: pos is NULL", what);
        CHECK(check_rows_of(c, what, q, q_stride, qk->n_heads, qk->head_dim, qk->x_dtype));
        CHECK(check_rows_of(c, what, dq, dq_stride, qk->n_heads, qk->head_dim, qk->x_dtype));
        CHECK(check_rows_of(c, what, dq_out, (long)qk->n_heads * qk->head_dim, qk->n_heads, qk->head_dim, qk->y_dtype));
        if (qk->n_kv_heads) {
            CHECK(check_rows_of(c, what, k, k_stride, qk->n_kv_heads, qk->head_dim, qk->x_dtype));
            CHECK(check_rows_of(c, what, dk, dk_stride, qk->n_kv_heads, qk->head_dim, qk->x_dtype));
            CHECK(check_rows_of(c, what, dk_out, (long)qk->n_kv_heads * qk->head_dim, qk->n_kv_heads, qk->head_dim, qk->y_dtype));
        }
        if (dq_gain || dk_gain) {
            if (!scratch) return ctx_fail(c, MRP_ERR_NULL, "%s: scratch is NULL", what);
            if (!aligned16(scratch)) return ctx_fail(c, MRP_ERR_ALIGN, "%s: scratch must be 16-byte aligned", what);
            if (scratch_bytes < mrp_qk_norm_rope_grad_scratch_bytes(n_rows, qk))
                return ctx_fail(c, MRP_ERR_WORKSPACE, "%s: scratch holds %zu of %zu bytes", what, scratch_bytes,
                                mrp_qk_norm_rope_grad_scratch_bytes(n_rows, qk));
        }
    }
    CHECK(check_device(c, what));
    hipStream_t st = static_cast<hipStream_t>(stream);
    QkGrad a;
    a.f = {*qk, n_rows, pos, q, k, q_stride, k_stride, const_cast<void *>(dq_out), const_cast<void *>(dk_out), ctx_view(c).err_flag};
    a.dq = dq; a.dk = dk; a.dq_stride = dq_stride; a.dk_stride = dk_stride;
    const int all = qk->n_heads + qk->n_kv_heads;
    a.wg_q = grad_workgroups(n_rows, qk->n_heads, all, qk->head_dim);
    a.wg_k = grad_workgroups(n_rows, qk->n_kv_heads, all, qk->head_dim);
    a.part = static_cast<float *>(scratch);
    a.dq_gain = dq_gain; a.dk_gain = dk_gain;
    if (n_rows > 0) {
        for_types(qk->x_dtype, qk->y_dtype, [&](auto xt, auto yt) {
            qk_norm_rope_grad_kernel<decltype(xt), decltype(yt)><<<a.wg_q + a.wg_k, 256, 0, st>>>(a);
        });
        CHECK(launched(c, what));
    }
    if (dq_gain || dk_gain) gain_sum_kernel<<<2 * (qk->head_dim / 16), 1024, 0, st>>>(a);
    return launched(c, what);
}

int mrp_cache_append(mrp_ctx *c, void *stream, long n_rows, const mrp_new_rows *rows, const mrp_qk *qk, const void *q, long q_stride,
                     const void *k, long k_stride, const void *v, long v_stride, const mrp_paged_cache *cache, void *q_out) {
    const char *what = "mrp_cache_append";
    if (!c) return MRP_ERR_NULL;
    if (!rows || !qk || !cache) return ctx_fail(c, MRP_ERR_NULL, "%s: NULL pointer", what);
    CHECK(check_qk(c, what, n_rows, qk));
    CHECK(check_new_rows(c, what, n_rows, rows));
    CHECK(check_cache(c, what, cache, rows->B));
    if (qk->head_dim != cache->head_dim || qk->n_kv_heads != cache->n_kv_heads)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d key heads of %d, but the cache has %d of %d", what, qk->n_kv_heads, qk->head_dim,
                        cache->n_kv_heads, cache->head_dim);
    if (n_rows == 0 || rows->B == 0) return MRP_OK;
    if (q) {
        if (qk->n_heads % qk->n_kv_heads) return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d heads over %d key heads", what, qk->n_heads, qk->n_kv_heads);
        CHECK(check_rows_of(c, what, q, q_stride, qk->n_heads, qk->head_dim, qk->x_dtype));
        CHECK(check_rows_of(c, what, q_out, (long)qk->n_heads * qk->head_dim, qk->n_heads, qk->head_dim, qk->y_dtype));
    }
    CHECK(check_rows_of(c, what, k, k_stride, qk->n_kv_heads, qk->head_dim, qk->x_dtype));
    CHECK(check_rows_of(c, what, v, v_stride, qk->n_kv_heads, qk->head_dim, qk->x_dtype));
    CHECK(check_device(c, what));
    const Append a = {*qk, *rows, *cache, (int)n_rows, q, k, v, q_stride, k_stride, v_stride, q_out, ctx_view(c).err_flag};
    const long threads = n_rows * ((q ? qk->n_heads : 0) + 2 * qk->n_kv_heads) * (qk->head_dim / 16);
    for_types(qk->x_dtype, qk->y_dtype, [&](auto xt, auto yt) {
        cache_append_kernel<decltype(xt), decltype(yt)><<<(unsigned)((threads + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(a);
    });
    return launched(c, what);
}

}  // extern "C"
