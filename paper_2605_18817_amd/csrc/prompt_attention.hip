// Attention over a paged cache for many rows of a key head: prompts and long blocks.
//
// The mathematics is that of paged_attention.hip, bounded by the matrix cores instead of the memory: 4 flops per row, position and
// entry.  A workgroup takes 32 rows for each of its waves (row r = token r / G, head r % G, so that all heads that share a key head read
// a tile of keys once) and walks the positions 64 at a time.  Keys and values come through shared memory, in two buffers: while a
// tile is worked on, the next one is on its way to registers.
//     S^T = K Q^T     (32x32x16: A = 32 keys x 16 entries, B = 16 entries x 32 rows, which stay in registers)
//     O^T += V^T P^T  (A = 32 entries x 16 keys, B = 16 keys x 32 rows)
// The result of the first product has keys 8 (i / 4) + 4 h + i % 4 of row r in registers i of lane 32 h + r, the second wants keys 8 h ..
// 8 h + 7 of every 16: a tile's keys lie in shared memory in the order that makes these the same, and the weights stay in
// their lanes.  Values are turned on their way into shared memory: entry d of all keys in row 'd / 2, odd entries behind the even
// ones', so that a lane ends up with neighbouring entries of its output row.
#include "paged_attention.h"

namespace mrp {

namespace {

constexpr int KT = 64;       // positions of a tile

__device__ __forceinline__ f32x16 mfma32(BF16, u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(F16, u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

struct Cut {
    int tiles;       // row tiles that a sequence can have
    int pieces;      // parts of the positions, joined by a second kernel where there is more than one
};

// Place of key x (0 .. 31) of a tile's half in shared memory
__device__ __forceinline__ int key_row(int x) {
    const int i = 8 * (x >> 4) + (x & 7), h = (x >> 3) & 1;
    return 8 * (i >> 2) + 4 * h + (i & 3);
}

// The tiles of a piece of a row tile
struct Piece {
    Steps st;
    int begin, end;
};
__device__ __forceinline__ Piece piece_of(const Attend &A, const SeqRows &s, int row0, int rows, int nr, int pieces, int piece) {
    Piece p;
    const int last = row0 + rows < nr ? row0 + rows - 1 : nr - 1;
    p.st = steps_of<KT>(A.attn, s.len - s.n + row0 / A.G, s.len - s.n + last / A.G, s.len);
    p.begin = (int)((long)p.st.steps * piece / pieces);
    p.end = (int)((long)p.st.steps * (piece + 1) / pieces);
    return p;
}

// LOADS of W bytes
template <int W>
__device__ __forceinline__ uint32_t load_part(const char *p) {
    if constexpr (W == 4) return *reinterpret_cast<const uint32_t *>(p);
    else return *reinterpret_cast<const uint16_t *>(p);
}

template <typename T, bool E8, int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void prompt_attention_kernel(const Attend A, const Cut P, float *scratch) {
    constexpr int ES = E8 ? 1 : 2, THREADS = 64 * NW, ROWS = 32 * NW;
    constexpr int NC = HD / 16;                   // contraction steps of a score
    constexpr int ND = HD / 32;                   // tiles of 32 entries of the output
    constexpr int KROW = HD * 2 + 16;             // bytes of a key's row in shared memory: 16 more spread the rows over the banks
    constexpr int VROW = KT * 2 + 16;             // ... and of an entry's
    constexpr int KP = HD * ES / 16;              // 16-byte pieces of a key
    constexpr int KN = KT * KP < THREADS ? 1 : KT * KP / THREADS;   // of them for a thread
    constexpr bool K_ALL = KT * KP >= THREADS;    // ... for every thread
    constexpr int DW = E8 ? 4 : 2;                // entries of a value that a thread takes
    constexpr int VL = HD / DW;                   // threads on a value
    constexpr int VK = KT * VL / THREADS;         // keys of a thread
    static_assert(VK >= 2 && VK <= 16, "a thread's share");
    __shared__ __align__(16) char ks[2][KT * KROW];
    __shared__ __align__(16) char vs[2][HD * VROW];
    __shared__ int slots[4][KT];                  // places of the positions of four tiles, -1: not there
    __shared__ uint32_t there[4][2];
    __shared__ int odd[4];                        // the tile has values that are not finite where only some rows see them

    const mrp_paged_cache &C = A.cache;
    const long cap = (long)C.max_pages * C.page_size;
    if (blockIdx.x == 0 && blockIdx.y == 0) check_rows(A.rows, A.n_rows, cap, A.err_flag, THREADS);
    // key heads side by side: with eight of them, an XCD's L2 serves one.  The last rows, which have the most to do, come first.
    const int kvh = blockIdx.x % C.n_kv_heads, rest = blockIdx.x / C.n_kv_heads, b = blockIdx.y, G = A.G;
    const SeqRows s = seq_rows(A.rows, A.n_rows, cap, b);
    const int nr = s.n * G, tiles = (nr + ROWS - 1) / ROWS;
    const int piece = rest % P.pieces, tile = tiles - 1 - rest / P.pieces;
    if (tile < 0) return;
    const int row0 = tile * ROWS;
    const Piece pc = piece_of(A, s, row0, ROWS, nr, P.pieces, piece);
    const Steps &st = pc.st;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r32 = lane & 31, h = lane >> 5;

    // the row's position and operand (lanes past the last row take it again and store nothing)
    const int my = row0 + 32 * wave + r32, r = my < nr ? my : nr - 1;
    const int tok = r / G, pos = s.len - s.n + tok, head = kvh * G + r - tok * G;
    u32x4 qf[NC];
    {
        const uint16_t *qp = A.q + (long)(s.begin + tok) * A.q_stride + (long)head * HD + 8 * h;
#pragma unroll
        for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const u32x4 *>(qp + 16 * c);
    }
    // what all rows see
    const int p_first = s.len - s.n + row0 / G, p_last = s.len - s.n + (row0 + ROWS < nr ? row0 + ROWS - 1 : nr - 1) / G, W = A.attn.window;
    const int full_high = p_first < 0 ? 0 : (A.attn.causal ? p_first + 1 : s.len);
    const int full_low = W && p_last + 1 > W ? p_last + 1 - W : 0;
    const int sink = A.attn.n_sink;

    const float c2 = A.attn.scale * 1.4426950408889634f * (E8 && C.k_scale ? C.k_scale[kvh] : 1.f);
    const long pitch = (long)C.n_kv_heads * HD * ES;
    const char *kb = static_cast<const char *>(C.k_pages) + (long)kvh * HD * ES;
    const char *vb = static_cast<const char *>(C.v_pages) + (long)kvh * HD * ES;
    const int32_t *table = C.page_table + (size_t)b * C.max_pages;

    auto key_of = [&](int u) { return (u < st.s_steps ? u : st.first + u - st.s_steps) * KT; };
    auto is_partial = [&](int key0, uint32_t th0, uint32_t th1) {
        return (th0 & th1) != 0xffffffffu || key0 + KT > full_high || (key0 < full_low && key0 + KT > sink);
    };
    // the first wave looks up the places of the piece's tile i
    auto look_up = [&](int i) {
        const int u = pc.begin + i, at = i & 3;
        if (wave == 0) {
            const int j = key_of(u) + lane;
            int slot = -1;
            if (j < st.high) {
                const int page = table[j / C.page_size];
                if (page >= 0 && page < C.n_pages) slot = page * C.page_size + j % C.page_size;
                else atomicOr(A.err_flag, ERR_PAGE);
            }
            slots[at][lane] = slot;
            const unsigned long long ok = __ballot(slot >= 0);
            if (lane == 0) {
                there[at][0] = (uint32_t)ok;
                there[at][1] = (uint32_t)(ok >> 32);
                odd[at] = 0;
            }
        }
    };
    uint4 kreg[KN];
    uint32_t vreg[VK];
    const int vd = tid % VL, vg = tid / VL;       // the thread's entries DW vd .., keys VK vg ..
    auto request = [&](int i) {
        const int at = i & 3;
#pragma unroll
        for (int n = 0; n < KN && (K_ALL || tid < KT * KP); ++n) {
            const int key = (tid + n * THREADS) / KP, part = (tid + n * THREADS) % KP, slot = slots[at][key];
            kreg[n] = *reinterpret_cast<const uint4 *>(kb + (slot < 0 ? 0 : slot) * pitch + 16 * part);
        }
#pragma unroll
        for (int n = 0; n < VK; ++n) {
            const int slot = slots[at][VK * vg + n];
            vreg[n] = load_part<DW * ES>(vb + (slot < 0 ? 0 : slot) * pitch + DW * ES * vd);
        }
    };
    auto put = [&](int i) {
        const int u = pc.begin + i, buf = i & 1, at = i & 3;
#pragma unroll
        for (int n = 0; n < KN && (K_ALL || tid < KT * KP); ++n) {
            const int key = (tid + n * THREADS) / KP, part = (tid + n * THREADS) % KP;
            char *to = ks[buf] + ((key & 32) + key_row(key & 31)) * KROW;
            if constexpr (E8) {
                uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
                widen(T{}, kreg[n].x, a0, a1);
                widen(T{}, kreg[n].y, a2, a3);
                widen(T{}, kreg[n].z, b0, b1);
                widen(T{}, kreg[n].w, b2, b3);
                reinterpret_cast<uint4 *>(to + 32 * part)[0] = make_uint4(a0, a1, a2, a3);
                reinterpret_cast<uint4 *>(to + 32 * part)[1] = make_uint4(b0, b1, b2, b3);
            } else {
                *reinterpret_cast<uint4 *>(to + 16 * part) = kreg[n];
            }
        }
        uint32_t w[VK][DW / 2];
#pragma unroll
        for (int n = 0; n < VK; ++n) {
            if constexpr (E8) widen(T{}, vreg[n], w[n][0], w[n][DW / 2 - 1]);
            else w[n][0] = vreg[n];
        }
        const int key0 = key_of(u);
        const uint32_t th0 = there[at][0], th1 = there[at][1];
        if (is_partial(key0, th0, th1)) {
            // values that no row sees are cleared; those that only some rows see and are not finite too, and the tile is marked
            bool bad = false;
#pragma unroll
            for (int n = 0; n < VK; ++n) {
                const int k = VK * vg + n, j = key0 + k;
                const bool any = j < st.high && (j >= st.low || j < sink) && (((k & 32 ? th1 : th0) >> (k & 31)) & 1u);
#pragma unroll
                for (int i = 0; i < DW / 2; ++i) {
                    const uint32_t v = any ? w[n][i] : 0u;
                    bad |= not_finite(T{}, v);
                    w[n][i] = finite_halves(T{}, v);
                }
            }
            if (bad) odd[at] = 1;
        }
#pragma unroll
        for (int e = 0; e < DW; ++e) {
            uint32_t col[VK / 2];
#pragma unroll
            for (int n = 0; n < VK / 2; ++n) col[n] = __builtin_amdgcn_perm(w[2 * n + 1][e / 2], w[2 * n][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            const int d = DW * vd + e;
            char *to = vs[buf] + ((d & 1) * (HD / 2) + (d >> 1)) * VROW + 2 * VK * vg;
            if constexpr (VK == 16) {
                reinterpret_cast<uint4 *>(to)[0] = make_uint4(col[0], col[1], col[2], col[3]);
                reinterpret_cast<uint4 *>(to)[1] = make_uint4(col[4], col[5], col[6], col[7]);
            } else if constexpr (VK == 8) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(col[0], col[1], col[2], col[3]);
            } else if constexpr (VK == 4) {
                *reinterpret_cast<uint2 *>(to) = make_uint2(col[0], col[1]);
            } else {
                *reinterpret_cast<uint32_t *>(to) = col[0];
            }
        }
    };

    float m = -INFINITY, l = 0.f;                 // m: reference of the sums, at most 8 below the largest score (in units of log 2)
    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;

    auto compute = [&](int i) {
        const int u = pc.begin + i, buf = i & 1, at = i & 3;
        const int key0 = key_of(u);
        const uint32_t th0 = there[at][0], th1 = there[at][1];
        f32x16 sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[t][i] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const u32x4 a = *reinterpret_cast<const u32x4 *>(ks[buf] + (32 * t + r32) * KROW + 32 * c + 16 * h);
                sc[t] = mfma32(T{}, a, qf[c], sc[t]);
            }
        }
        const bool partial = is_partial(key0, th0, th1);
        if (partial) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t seen = (seen_bits(pos, key0 + 32 * t, s.len, A.attn) & (t ? th1 : th0)) >> (8 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][i] = (seen >> (16 * (i >> 3) + (i & 7))) & 1u ? sc[t][i] : -INFINITY;
            }
        }
        float mx = sc[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) mx = fmaxf(mx, sc[i >> 4][i & 15]);
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        // the sums are brought to a new reference where a score is more than a factor of 2^8 above the old one
        if (__any((mx - m) * c2 > 8.f || (m == -INFINITY && mx > m))) {
            const float top = fmaxf(m, mx);
            const float alpha = m == -INFINITY ? 0.f : exp2f((m - top) * c2);
            m = top;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] *= alpha;
        }
        const float ref = m == -INFINITY ? 0.f : m * c2;
        u32x4 p[4];                               // the weights of 16 keys each, rounded to 16 bits
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float p0 = exp2f(fmaf(sc[i >> 4][i & 15], c2, -ref)), p1 = exp2f(fmaf(sc[i >> 4][(i & 15) + 1], c2, -ref));
            float x, y;
            sum += p0 + p1;
            p[i >> 3][(i & 7) >> 1] = pack2(T{}, p0, p1, x, y);
        }
        l += sum;
        if (partial && odd[at]) {
            // add what is not finite to the rows that see it, from the cache itself
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll 1
                    for (int hh = 0; hh < 2; ++hh) {
                        const int k = 16 * q + 8 * hh + j, slot = slots[at][k];
                        const uint32_t two = __shfl(p[q][j / 2], 32 * hh + r32);
                        const float weight = to_float(T{}, j & 1 ? two >> 16 : two & 0xffffu);
                        const bool sees = slot >= 0 && ((seen_bits(pos, key0 + (k & 32), s.len, A.attn) >> (k & 31)) & 1u);
                        if (!sees) continue;
#pragma unroll
                        for (int d = 0; d < ND; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int x = 32 * d + 8 * (i >> 2) + 4 * h + (i & 3), e = 2 * (x % (HD / 2)) + x / (HD / 2);
                                uint32_t half;
                                if constexpr (E8) {
                                    uint32_t lo, hi;
                                    widen(T{}, *reinterpret_cast<const uint8_t *>(vb + slot * pitch + e), lo, hi);
                                    half = lo & 0xffffu;
                                } else {
                                    half = *reinterpret_cast<const uint16_t *>(vb + slot * pitch + 2 * e);
                                }
                                if (not_finite(T{}, half)) acc[d][i] += weight * to_float(T{}, half);
                            }
                    }
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x4 a = *reinterpret_cast<const u32x4 *>(vs[buf] + (32 * d + r32) * VROW + 32 * q + 16 * h);
                acc[d] = mfma32(T{}, a, p[q], acc[d]);
            }
    };

    // three tiles are on their way: the places of the one after the next, keys and values of the next, and the one at work
    const int n = pc.end - pc.begin;
    if (n > 0) {
        look_up(0);
        if (n > 1) look_up(1);
        __syncthreads();
        request(0);
        put(0);
        __syncthreads();
    }
    for (int i = 0; i < n; ++i) {
        if (i + 1 < n) request(i + 1);
        if (i + 2 < n) look_up(i + 2);
        compute(i);
        if (i + 1 < n) put(i + 1);
        __syncthreads();
    }

    l += __shfl_xor(l, 32);
    if (my >= nr) return;
    const bool empty = m == -INFINITY;
    const float v_scale = E8 && C.v_scale ? C.v_scale[kvh] : 1.f;
    if (P.pieces > 1) {
        float *place = scratch + (((size_t)b * P.tiles + tile) * C.n_kv_heads + kvh) * P.pieces * ROWS * (HD + 2) + (size_t)piece * ROWS * (HD + 2);
        float *dst = place + (size_t)(32 * wave + r32) * HD;
#pragma unroll
        for (int d = 0; d < ND / 2; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                float4 *to = reinterpret_cast<float4 *>(dst + 2 * (32 * d + 2 * i + 4 * h));
                to[0] = make_float4(acc[d][i], acc[d + ND / 2][i], acc[d][i + 1], acc[d + ND / 2][i + 1]);
                to[1] = make_float4(acc[d][i + 2], acc[d + ND / 2][i + 2], acc[d][i + 3], acc[d + ND / 2][i + 3]);
            }
        if (h == 0) *reinterpret_cast<float2 *>(place + (size_t)ROWS * HD + 2 * (32 * wave + r32)) = make_float2(m, l);
        return;
    }
    const long at = (long)(s.begin + tok) * A.attn.n_heads + head;
    const float f = empty ? 0.f : v_scale / l;
#pragma unroll
    for (int d = 0; d < ND / 2; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            uint32_t w[4];
            float x, y;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = empty ? 0u : pack2(T{}, acc[d][i + k] * f, acc[d + ND / 2][i + k] * f, x, y);
            *reinterpret_cast<uint4 *>(A.out + at * HD + 2 * (32 * d + 2 * i + 4 * h)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    if (A.lse && h == 0) A.lse[at] = empty ? -INFINITY : m * c2 * 0.6931471805599453f + logf(l);
}

// Adds up a row tile's pieces in the order of their positions: 16 threads a row, 16 rows a workgroup
template <typename T, bool E8, int HD, int NW>
__global__ __launch_bounds__(256) void prompt_join_kernel(const Attend A, const Cut P, const float *scratch) {
    constexpr int ROWS = 32 * NW, NE = HD / 16;
    const mrp_paged_cache &C = A.cache;
    const int per = ROWS / 16, b = blockIdx.y, slice = blockIdx.x % per, kvh = blockIdx.x / per % C.n_kv_heads, tile = blockIdx.x / per / C.n_kv_heads;
    const SeqRows s = seq_rows(A.rows, A.n_rows, (long)C.max_pages * C.page_size, b);
    const int rr = 16 * slice + (threadIdx.x >> 4), part = threadIdx.x & 15, r = tile * ROWS + rr;
    if (r >= s.n * A.G) return;
    const float c2 = A.attn.scale * 1.4426950408889634f * (E8 && C.k_scale ? C.k_scale[kvh] : 1.f);
    const float *place = scratch + (((size_t)b * P.tiles + tile) * C.n_kv_heads + kvh) * P.pieces * ROWS * (HD + 2);
    float mx = -INFINITY, sum = 0.f, o[NE];
    for (int q = 0; q < P.pieces; ++q) mx = fmaxf(mx, place[(size_t)q * ROWS * (HD + 2) + (size_t)ROWS * HD + 2 * rr]);
#pragma unroll
    for (int e = 0; e < NE; ++e) o[e] = 0.f;
    for (int q = 0; q < P.pieces; ++q) {
        const float *p = place + (size_t)q * ROWS * (HD + 2);
        const float2 ml = *reinterpret_cast<const float2 *>(p + (size_t)ROWS * HD + 2 * rr);
        const float f = ml.x == -INFINITY ? 0.f : exp2f((ml.x - mx) * c2);
        sum += f * ml.y;
        const float4 *src = reinterpret_cast<const float4 *>(p + (size_t)rr * HD + NE * part);
#pragma unroll
        for (int e = 0; e < NE; e += 4) {
            const float4 v = src[e / 4];
            o[e] += f * v.x; o[e + 1] += f * v.y; o[e + 2] += f * v.z; o[e + 3] += f * v.w;
        }
    }
    const int t = r / A.G;
    store_row<T, HD>(A, s.begin + t, kvh * A.G + r - t * A.G, part, mx == -INFINITY, mx * c2, sum, E8 && C.v_scale ? C.v_scale[kvh] : 1.f, o);
}

// Waves of a workgroup: four where a sequence has no more than 128 rows of a key head
int waves_for(long rows) { return rows <= 128 ? 4 : 8; }

// Pieces: as many as find a compute unit each, while a piece keeps four tiles of the longest sequence that the table allows
Cut cut_of(long rows, int B, int n_kv_heads, long positions, int nCU) {
    Cut c;
    const int per = 32 * waves_for(rows);
    c.tiles = (int)((rows + per - 1) / per);
    const long items = (long)c.tiles * B * n_kv_heads, longest = positions / (4 * KT);
    long pieces = items > 0 ? nCU / items : 1;
    if (pieces > longest) pieces = longest;
    c.pieces = pieces < 1 ? 1 : (int)pieces;
    return c;
}

template <typename T, bool E8, int HD, int NW>
void launch(const Attend &a, const Cut &c, float *scratch, hipStream_t st) {
    prompt_attention_kernel<T, E8, HD, NW><<<dim3(c.tiles * a.cache.n_kv_heads * c.pieces, a.rows.B), 64 * NW, 0, st>>>(a, c, scratch);
    if (c.pieces > 1)
        prompt_join_kernel<T, E8, HD, NW><<<dim3(c.tiles * a.cache.n_kv_heads * (2 * NW), a.rows.B), 256, 0, st>>>(a, c, scratch);
}

template <typename T, bool E8>
void launch_form(const Attend &a, const Cut &c, int waves, float *scratch, hipStream_t st) {
    if (a.cache.head_dim == 64) waves == 4 ? launch<T, E8, 64, 4>(a, c, scratch, st) : launch<T, E8, 64, 8>(a, c, scratch, st);
    else waves == 4 ? launch<T, E8, 128, 4>(a, c, scratch, st) : launch<T, E8, 128, 8>(a, c, scratch, st);
}

}  // namespace

bool prompt_takes(long rows, int head_dim) { return rows > 64 && head_dim <= 128; }

size_t prompt_scratch_floats(long rows, int B, int n_kv_heads, long positions, int head_dim, int nCU) {
    const Cut c = cut_of(rows, B, n_kv_heads, positions, nCU);
    return c.pieces > 1 ? (size_t)c.tiles * B * n_kv_heads * c.pieces * 32 * waves_for(rows) * (head_dim + 2) : 0;
}

hipError_t launch_prompt_attention(const Attend &a, float *scratch, int nCU, hipStream_t st) {
    const long rows = most_rows(a.n_rows, a.rows, a.G);
    const Cut c = cut_of(rows, a.rows.B, a.cache.n_kv_heads, (long)a.cache.max_pages * a.cache.page_size, nCU);
    const bool e8 = a.cache.dtype == MRP_DTYPE_E4M3;
    if (a.attn.dtype == MRP_DTYPE_BF16) e8 ? launch_form<BF16, true>(a, c, waves_for(rows), scratch, st) : launch_form<BF16, false>(a, c, waves_for(rows), scratch, st);
    else e8 ? launch_form<F16, true>(a, c, waves_for(rows), scratch, st) : launch_form<F16, false>(a, c, waves_for(rows), scratch, st);
    return hipGetLastError();
}

}  // namespace mrp
