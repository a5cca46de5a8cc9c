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
//
// Bound by the memory: a wave asks for 16 KB a step (heads of 128, 16 bits) and two waves share a SIMD.  64 caches of up to 32767
// positions, 8 key heads of 128: 2.1 GB in 373 us, 5.7 TB/s (pages of one position 5.3); of 8 bits 4.5, whose 128 bytes a position lie
// 1 KB apart; of 64 entries, 12 key heads, 4.9.
#include "paged_attention.h"

namespace mrp {

int check_new_rows(mrp_ctx *c, const char *what, long n_rows, const mrp_new_rows *r);
int check_cache(mrp_ctx *c, const char *what, const mrp_paged_cache *k, int B);
int check_context_device(mrp_ctx *c, const char *what);

namespace {

constexpr int WAVES = 4;
constexpr int STEP = 32;     // positions per step of a wave

// ---- how the work is split
//
// A sequence's steps come in units of WAVES, and units(b) counts those that any of its rows needs.  Its items, one for each key
// head and tile of 16 RT rows, take that many units each, and the units of all items of all sequences, in order, are cut
// into as many equal ranges as there are workgroups.  A range that ends inside an item leaves a partial result (sums, their reference m, and
// l) in one of the workgroup's two places: place 1 if it has the item's first unit, place 0 otherwise; an item's pieces are then
// added up in order by a second kernel.  Nothing is planned on the host, which does not know the lengths.
struct Split {
    int rows;          // rows of a tile
    int tiles;         // of them that a sequence can have
    int workgroups;    // at most
};
// What the workgroup with an item's first unit notes of it: itself, and over how many workgroups the item goes
struct Pieces {
    int first, count;
};

__device__ __forceinline__ int units_of(const Attend &A, const SeqRows &s) {
    const int u = (steps_of<STEP>(A.attn, s.len - s.n, s.len - 1, s.len).steps + WAVES - 1) / WAVES;
    return u > 1 ? u : 1;
}
__device__ __forceinline__ long cost_of(const Attend &A, const Split &P, const SeqRows &s) {
    return s.n ? (long)A.cache.n_kv_heads * ((s.n * A.G + P.rows - 1) / P.rows) * units_of(A, s) : 0;
}
// x / y for 0 <= x < 2^52, 0 < y: the quotient of doubles is off by less than one
__device__ __forceinline__ long quotient(long x, long y) {
    long q = (long)((double)x / (double)y);
    if (q * y > x) --q;
    else if ((q + 1) * y <= x) ++q;
    return q;
}
// n ranges of `size` units, the first `longer` of one more
struct Ranges {
    int n;
    long size, longer;
    __device__ long begin(int w) const { return size * w + (w < longer ? w : longer); }
};
__device__ __forceinline__ Ranges ranges_of(const Split &P, long total) {
    Ranges r;
    r.n = total < 1 ? 1 : (total < P.workgroups ? (int)total : P.workgroups);
    r.size = quotient(total, r.n);
    r.longer = total - r.size * r.n;
    return r;
}

// partial results: per workgroup and place `rows` x (HD sums), then `rows` x (m, l)
__host__ __device__ constexpr size_t place_floats(int rows, int HD) { return (size_t)rows * (HD + 2); }

// RG: the waves of a workgroup are RG groups with 16 rows each, and those of a group take the steps in turn (waves of two groups
// ask for the same keys and values, which come from memory once)
template <typename T, bool E8, int HD, int RG>
__global__ __launch_bounds__(64 * WAVES, HD <= 128 ? 2 : 1) void paged_attention_kernel(const Attend A, const Split P, float *scratch, Pieces *items) {
    constexpr int ES = E8 ? 1 : 2;             // bytes of a cache entry
    constexpr int NC = HD / 32;                // contraction steps of a score
    constexpr int NE = HD / 16;                // entries of a lane's share of V, and A operands of O^T
    constexpr int NL = E8 ? NC / 2 : NC;       // 16-byte pieces of a lane's share of K
    constexpr int WK = WAVES / RG;             // waves of a group
    constexpr int TILE = 16 * RG;              // rows of a workgroup
    // A step's keys and values are asked for a turn ahead where they fit the registers twice (64 caches of up to 32767 positions of 8
    // bits: 257 us without, 238 with it; 16 bits, 12 heads of 64: 325 without, 345 with it: two waves of a SIMD cover for each other)
    constexpr bool AHEAD = E8 && HD <= 128;
    __shared__ float sm[WAVES][16], sl[WAVES][16];
    __shared__ __align__(16) float so[WAVES][16][HD + 4];
    __shared__ long scan[WAVES];
    __shared__ long seq_base;
    __shared__ int seq_at;
    __shared__ SeqRows seq_of;

    const mrp_paged_cache &C = A.cache;
    const long cap = (long)C.max_pages * C.page_size;
    if (blockIdx.x == 0) check_rows(A.rows, A.n_rows, cap, A.err_flag, 64 * WAVES);

    // this workgroup's range, and the sequence that it begins in
    long cur, end, base, longer, size;
    int b;
    {
        const int per = (A.rows.B + 64 * WAVES - 1) / (64 * WAVES), b0 = threadIdx.x * per;
        long mine = 0;
        for (int i = b0; i < b0 + per && i < A.rows.B; ++i) mine += cost_of(A, P, seq_rows(A.rows, A.n_rows, cap, i));
        long incl = mine;
        for (int off = 1; off < 64; off <<= 1) {
            const long y = __shfl_up(incl, off);
            if ((threadIdx.x & 63) >= off) incl += y;
        }
        if ((threadIdx.x & 63) == 63) scan[threadIdx.x >> 6] = incl;
        __syncthreads();
        long before = 0, total = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < (int)(threadIdx.x >> 6)) before += scan[w];
            total += scan[w];
        }
        const Ranges all = ranges_of(P, total);
        if ((int)blockIdx.x >= all.n) return;
        cur = all.begin(blockIdx.x);
        end = all.begin(blockIdx.x + 1);
        longer = all.longer;
        size = all.size;
        if (cur >= end) return;
        long at = before + incl - mine;
        if (at <= cur && cur < at + mine) {
            int i = b0;
            SeqRows s;
            for (;; ++i) {
                s = seq_rows(A.rows, A.n_rows, cap, i);
                const long c = cost_of(A, P, s);
                if (cur < at + c) break;
                at += c;
            }
            seq_at = i;
            seq_base = at;
            seq_of = s;
        }
        __syncthreads();
        b = seq_at;
        base = seq_base;
    }
    SeqRows s = seq_of;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4, G = A.G;
    const int group = wave % RG, turn = wave / RG;
    const long pitch = (long)C.n_kv_heads * HD * ES;      // bytes between positions
    const bool whole = C.page_size % STEP == 0;           // a step lies in one page
    const bool causal = A.attn.causal != 0;
    const int W = A.attn.window, sink = A.attn.n_sink;

    for (;; s = seq_rows(A.rows, A.n_rows, cap, ++b)) {   // sequences
        const long cost = cost_of(A, P, s);
        if (cost == 0) continue;
        const int units = units_of(A, s), nr = s.n * G, tiles = (nr + P.rows - 1) / P.rows;
        const int32_t *table = C.page_table + (size_t)b * C.max_pages;
        while (cur < base + cost && cur < end) {          // items
            const long item = (cur - base) / units;
            const int unit0 = (int)(cur - base - item * units), unit1 = units - unit0 <= end - cur ? units : unit0 + (int)(end - cur);
            const int kvh = (int)(item / tiles), row0 = (int)(item % tiles) * P.rows;
            if (unit0 == 0 && threadIdx.x == 0) {
                int count = 1;
                for (long at = end, w = blockIdx.x + 1; at < cur + units; ++w, ++count) at += size + (w < longer);
                items[((size_t)b * P.tiles + item % tiles) * C.n_kv_heads + kvh] = Pieces{(int)blockIdx.x, count};
            }
            cur += unit1 - unit0;
            __syncthreads();                               // (the item before has been read out of shared memory)

            // the rows' positions and operands; lanes past the last row take it again and store nothing
            int pos;
            u32x4 qf[NC];
            const int mine0 = row0 + 16 * group;      // the wave's first row
            const int r = mine0 + r16 < nr ? mine0 + r16 : nr - 1;
            const int t = r / G;
            pos = s.len - s.n + t;
            const uint16_t *qp = A.q + (long)(s.begin + t) * A.q_stride + (long)(kvh * G + r - t * G) * HD;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                // (8 bits: a lane's 16 bytes are 16 entries, for two contraction steps)
                const int at = E8 ? 64 * (c >> 1) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
                qf[c] = *reinterpret_cast<const u32x4 *>(qp + at);
            }

            // positions that any row of the workgroup sees: [0, sink) and [low, high); [full_low, full_high) is what all of the wave's see
            auto pos_of = [&](int r) { return s.len - s.n + (r < nr ? r : nr - 1) / G; };
            const Steps st = steps_of<STEP>(A.attn, pos_of(row0), pos_of(row0 + TILE - 1), s.len);
            const int low = st.low, high = st.high, p_first = pos_of(mine0), p_last = pos_of(mine0 + 15);
            const int full_high = p_first < 0 ? 0 : (causal ? p_first + 1 : s.len);
            const int full_low = W && p_last + 1 > W ? p_last + 1 - W : 0;
            const int step_end = mine0 >= nr ? 0 : (st.steps < unit1 * WAVES ? st.steps : unit1 * WAVES);

            const float c2 = A.attn.scale * 1.4426950408889634f * (E8 && C.k_scale ? C.k_scale[kvh] : 1.f);
            const char *kb = static_cast<const char *>(C.k_pages) + (long)kvh * HD * ES;
            const char *vb = static_cast<const char *>(C.v_pages) + (long)kvh * HD * ES;

            float m, l;
            f32x4 acc[NE];
            m = -INFINITY;
            l = 0.f;
#pragma unroll
            for (int e = 0; e < NE; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};

            auto key_of = [&](int u) { return (u < st.s_steps ? u : st.first + u - st.s_steps) * STEP; };
            // the page of step u's positions (of position key + lane % 32, where pages end inside a step; 0 where no row sees it)
            auto page_of = [&](int u) {
                const int j = key_of(u) + (whole ? 0 : (lane & 31));
                return j < high && (whole || j >= low || j < sink) ? table[j / C.page_size] : 0;
            };
            struct Raw {
                u32x4 k[2][NL];
                Words<NE * ES / 4> v[8];
                uint32_t there;                // positions whose page is there
            };
            // requests step u's keys and values: the lane's share of K, entries of two positions, and of V, entries NE r16 .. of
            // positions key0 + 8 g .. + 7
            auto request = [&](int u, int page, Raw &f) {
                const int key0 = key_of(u);
                const bool ok = page >= 0 && page < C.n_pages;
                if (!ok) atomicOr(A.err_flag, ERR_PAGE);
                if (whole) {
                    f.there = ok ? 0xffffffffu : 0u;
                    if (!ok) return;
                    const long at = ((long)page * C.page_size + key0 % C.page_size) * pitch;
                    const char *kp = kb + at + (int)(8 * (r16 >> 2) + (r16 & 3)) * pitch + 16 * g, *vp = vb + at + 8 * g * pitch + NE * ES * r16;
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int c = 0; c < NL; ++c) f.k[t][c] = load_16<RG == 1>(kp + 4 * t * pitch + 64 * c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f.v[j] = load_words<NE * ES / 4, RG == 1>(vp + j * pitch);
                } else {
                    const int j0 = key0 + (lane & 31);
                    const int slot = ok && j0 < high ? page * C.page_size + j0 % C.page_size : 0;
                    f.there = (uint32_t)__ballot(ok);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const char *kp = kb + __shfl(slot, 8 * (r16 >> 2) + 4 * t + (r16 & 3)) * pitch + 16 * g;
#pragma unroll
                        for (int c = 0; c < NL; ++c) f.k[t][c] = load_16<RG == 1>(kp + 64 * c);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) f.v[j] = load_words<NE * ES / 4, RG == 1>(vb + __shfl(slot, 8 * g + j) * pitch + NE * ES * r16);
                }
            };

            auto compute = [&](int u, const Raw &f) {
                const int key0 = key_of(u);
                const uint32_t there = f.there;
                if (there == 0) return;
                const bool partial = there != 0xffffffffu || key0 + STEP > full_high || (key0 < full_low && key0 + STEP > sink);
                f32x4 sc[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    u32x4 kf[NC];
                    if constexpr (E8) {
#pragma unroll
                        for (int c = 0; c < NL; ++c) {
                            uint32_t a0, a1, a2, a3;
                            widen(T{}, f.k[t][c][0], a0, a1);
                            widen(T{}, f.k[t][c][1], a2, a3);
                            kf[2 * c] = u32x4{a0, a1, a2, a3};
                            widen(T{}, f.k[t][c][2], a0, a1);
                            widen(T{}, f.k[t][c][3], a2, a3);
                            kf[2 * c + 1] = u32x4{a0, a1, a2, a3};
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < NC; ++c) kf[c] = f.k[t][c];
                    }
                    sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < NC; ++c) sc[t] = mfma(T{}, kf[c], qf[c], sc[t]);
                }
                uint32_t vw[8][NE / 2];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (E8) {
#pragma unroll
                        for (int w = 0; w < NE / 4; ++w) widen(T{}, f.v[j].w[w], vw[j][2 * w], vw[j][2 * w + 1]);
                    } else {
#pragma unroll
                        for (int w = 0; w < NE / 2; ++w) vw[j][w] = f.v[j].w[w];
                    }
                }

                float mx = fmaxf(m, LOWEST);
                if (partial) {
                    // scores of positions that a row does not see are dropped
                    const uint32_t all = seen_bits(pos, key0, s.len, A.attn) & there, seen = all >> (8 * g);
                    mx = all ? mx : m;
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sc[t][i] = (seen >> (4 * t + i)) & 1u ? sc[t][i] : -INFINITY;
                }

                // softmax of the step, and the weights as operands: the leading 16-bit term and the next
                u32x4 ph, pl;
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, fmaxf(sc[0][i], sc[1][i]));
                mx = max_halves(max_quarters(mx));
                const float shift = Few<T>::SHIFT - reference(mx, c2);
                if (__any(mx > m)) {
                    const float alpha = exp2_(shift - (Few<T>::SHIFT - reference(m, c2)));   // (exactly 1 where the row's maximum stays)
                    l *= alpha;
#pragma unroll
                    for (int e = 0; e < NE; ++e) acc[e] *= alpha;
                }
                m = mx;
                float sum = 0.f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const float p0 = exp2_(fmaf(sc[t][i], c2, shift)), p1 = exp2_(fmaf(sc[t][i + 1], c2, shift));
                        float r0, r1, x, y;
                        sum += p0 + p1;
                        ph[2 * t + i / 2] = pack2(T{}, p0, p1, r0, r1);
                        pl[2 * t + i / 2] = pack2(T{}, r0, r1, x, y);
                    }
                l += sum;

                bool bad = false;
                if (partial) {                     // values that no row sees are cleared
                    const uint32_t any = (first_bits(high - key0) & (~first_bits(low - key0) | first_bits(sink - key0)) & there) >> (8 * g);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int w = 0; w < NE / 2; ++w) {
                            vw[j][w] = (any >> j) & 1u ? vw[j][w] : 0u;
                            bad |= not_finite(T{}, vw[j][w]);
                        }
                    bad = __any(bad);
                }
                // entry e of the lanes' shares as an A operand
                auto turned = [&](int e) {
                    u32x4 vt;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        vt[k] = __builtin_amdgcn_perm(vw[2 * k + 1][e / 2], vw[2 * k][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
                    return vt;
                };
                if (bad) {
                    // A weight of zero times a value that is not finite is not zero.  Such values leave the product; how many of them a
                    // row sees in an entry is a product too, of ones, and makes the row's entry NaN
                    const uint32_t seen = seen_bits(pos, key0, s.len, A.attn) >> (8 * g);
                    u32x4 sees;
#pragma unroll
                    for (int j = 0; j < 4; ++j) sees[j] = ((seen >> (2 * j)) & 1u) * one_bits(T{}) + (((seen >> (2 * j + 1)) & 1u) * one_bits(T{}) << 16);
#pragma unroll
                    for (int e = 0; e < NE; ++e) {
                        u32x4 other = turned(e);
#pragma unroll
                        for (int k = 0; k < 4; ++k) other[k] = odd_halves(T{}, other[k]);
                        const f32x4 count = mfma(T{}, other, sees, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[e][i] = count[i] > 0.f ? NAN : acc[e][i];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int w = 0; w < NE / 2; ++w) vw[j][w] = finite_halves(T{}, vw[j][w]);
                }
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    const u32x4 vt = turned(e);
                    acc[e] = mfma(T{}, vt, ph, acc[e]);
                    acc[e] = mfma(T{}, vt, pl, acc[e]);
                }
            };

            {
                int u = unit0 * WAVES + turn;
                int page1 = u < step_end ? page_of(u) : 0, page2 = u + WK < step_end ? page_of(u + WK) : 0;
                if constexpr (AHEAD) {
                    Raw f;
                    if (u < step_end) request(u, page1, f);
                    for (; u < step_end; u += WK) {
                        Raw next;
                        const bool more = u + WK < step_end;
                        if (more) request(u + WK, page2, next);
                        if (u + 2 * WK < step_end) page2 = page_of(u + 2 * WK);
                        compute(u, f);
                        if (more) f = next;
                    }
                } else {
                    for (; u < step_end; u += WK) {
                        Raw f;
                        request(u, page1, f);
                        page1 = page2;
                        if (u + 2 * WK < step_end) page2 = page_of(u + 2 * WK);
                        compute(u, f);
                    }
                }
            }

            // the four lanes of a row add up their sums, the waves their rows
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (g == 0) {
                sm[wave][r16] = m;
                sl[wave][r16] = l;
            }
            const bool all = unit0 == 0 && unit1 == units;
            float *const place = all ? nullptr : scratch + ((size_t)blockIdx.x * 2 + (unit0 == 0 ? 1 : 0)) * place_floats(P.rows, HD);
            const float v_scale = E8 && C.v_scale ? C.v_scale[kvh] : 1.f;
            __syncthreads();
            {
                float mx = -INFINITY;
#pragma unroll
                for (int w = 0; w < WK; ++w) mx = fmaxf(mx, sm[group + RG * w][r16]);
                const float f = m == -INFINITY ? 0.f : exp2_((m - mx) * c2);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < NE; e += 4)
                        *reinterpret_cast<float4 *>(&so[wave][r16][NE * (4 * g + i) + e]) =
                            make_float4(acc[e][i] * f, acc[e + 1][i] * f, acc[e + 2][i] * f, acc[e + 3][i] * f);
            }
            __syncthreads();
            const int rr = threadIdx.x >> 4, part = threadIdx.x & 15;
#pragma unroll
            for (int q = 0; q < RG; ++q) {
                const int at = 16 * q + rr, r = row0 + at;
                if (r >= nr) break;
                float mx = -INFINITY, sum = 0.f;
#pragma unroll
                for (int w = 0; w < WK; ++w) mx = fmaxf(mx, sm[q + RG * w][rr]);
                float o[NE];
#pragma unroll
                for (int e = 0; e < NE; ++e) o[e] = 0.f;
#pragma unroll
                for (int w = 0; w < WK; ++w) {
                    const float mw = sm[q + RG * w][rr];
                    if (mw != -INFINITY) sum += sl[q + RG * w][rr] * exp2_((mw - mx) * c2);
#pragma unroll
                    for (int e = 0; e < NE; ++e) o[e] += so[q + RG * w][rr][NE * part + e];
                }
                if (all) {
                    const int t = r / G;
                    store_row<T, HD>(A, s.begin + t, kvh * G + r - t * G, part, mx == -INFINITY, mx * c2, Few<T>::ONE, sum, v_scale, o);
                } else {
                    float4 *dst = reinterpret_cast<float4 *>(place + (size_t)at * HD + NE * part);
#pragma unroll
                    for (int e = 0; e < NE; e += 4) dst[e / 4] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    if (part == 0) *reinterpret_cast<float2 *>(place + (size_t)P.rows * HD + 2 * at) = make_float2(mx, sum);
                }
            }
        }
        base += cost;
        if (cur >= end) return;
    }
}

// Adds up the pieces of an item that several workgroups had a part in, in the order of its positions: 16 threads a row
template <typename T, bool E8, int HD>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(const Attend A, const Split P, const float *scratch, const Pieces *items) {
    constexpr int NE = HD / 16;
    const mrp_paged_cache &C = A.cache;
    const int b = blockIdx.y, kvh = blockIdx.x % C.n_kv_heads, tile = blockIdx.x / C.n_kv_heads;
    const Pieces it = items[((size_t)b * P.tiles + tile) * C.n_kv_heads + kvh];   // (of no meaning where there is no such tile)
    const SeqRows s = seq_rows(A.rows, A.n_rows, (long)C.max_pages * C.page_size, b);
    const int nr = s.n * A.G, row0 = tile * P.rows, w0 = it.first, pieces = it.count;
    if (row0 >= nr || pieces == 1) return;
    const float c2 = A.attn.scale * 1.4426950408889634f * (E8 && C.k_scale ? C.k_scale[kvh] : 1.f);
    const float v_scale = E8 && C.v_scale ? C.v_scale[kvh] : 1.f;
    const size_t size = place_floats(P.rows, HD);
    const float *const first = scratch + (2 * (size_t)w0 + 1) * size, *const others = scratch + 2 * (size_t)w0 * size;
    const int rows = nr - row0 < P.rows ? nr - row0 : P.rows, part = threadIdx.x & 15;
    for (int rr = threadIdx.x >> 4; rr < rows; rr += 16) {
        // the row's 16 threads look at 16 pieces at a time
        auto sums = [&](int q) {
            return q < pieces ? *reinterpret_cast<const float2 *>((q ? others + 2 * (size_t)q * size : first) + (size_t)P.rows * HD + 2 * rr) : make_float2(-INFINITY, 0.f);
        };
        float mx = -INFINITY, sum = 0.f, o[NE];
        for (int q = part; q < pieces; q += 16) mx = fmaxf(mx, sums(q).x);
        for (int off = 1; off < 16; off <<= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
#pragma unroll
        for (int e = 0; e < NE; ++e) o[e] = 0.f;
        for (int q0 = 0; q0 < pieces; q0 += 16) {
            const float2 ml = sums(q0 + part);
            const float mine = ml.x == -INFINITY ? 0.f : exp2_((ml.x - mx) * c2);
            sum += mine * ml.y;
            const int count = pieces - q0 < 16 ? pieces - q0 : 16;
            for (int q1 = 0; q1 < count; q1 += 4) {      // (four requests at a time; past the end the last piece again, at a weight of zero)
                float4 v[4][NE / 4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int q = q0 + (q1 + x < count ? q1 + x : count - 1);
                    const float4 *src = reinterpret_cast<const float4 *>((q ? others + 2 * (size_t)q * size : first) + (size_t)rr * HD + NE * part);
#pragma unroll
                    for (int e = 0; e < NE / 4; ++e) v[x][e] = src[e];
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float f = q1 + x < count ? __shfl(mine, (threadIdx.x & 48) + q1 + x) : 0.f;
#pragma unroll
                    for (int e = 0; e < NE; e += 4) {
                        o[e] += f * v[x][e / 4].x; o[e + 1] += f * v[x][e / 4].y; o[e + 2] += f * v[x][e / 4].z; o[e + 3] += f * v[x][e / 4].w;
                    }
                }
            }
        }
        for (int off = 1; off < 16; off <<= 1) sum += __shfl_xor(sum, off);
        const int r = row0 + rr, t = r / A.G;
        store_row<T, HD>(A, s.begin + t, kvh * A.G + r - t * A.G, part, mx == -INFINITY, mx * c2, Few<T>::ONE, sum, v_scale, o);
    }
}

int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

// Rows of a workgroup: the fewest of 16, 32, 64 that hold a sequence's (more than 32 of up to 128 entries are not this kernel's).  The
// largest number of workgroups is what fits the device at once: two a compute unit, one for heads of 256.
Split split_of(long rows, int HD, int nCU) {
    const int tr = rows <= 16 ? 16 : (rows <= 32 ? 32 : 64);
    return Split{tr, ceil_div(rows, tr), (HD <= 128 ? 2 : 1) * (nCU > 0 ? nCU : 1)};
}
size_t partial_floats(const Split &p, int HD) { return 2 * (size_t)p.workgroups * place_floats(p.rows, HD); }

template <typename T, bool E8, int HD>
void launch(const Attend &a, const Split &p, float *scratch, hipStream_t st) {
    Pieces *const items = reinterpret_cast<Pieces *>(scratch + partial_floats(p, HD));
    if (p.rows == 16) paged_attention_kernel<T, E8, HD, 1><<<p.workgroups, 64 * WAVES, 0, st>>>(a, p, scratch, items);
    else if (HD <= 128 || p.rows == 32) paged_attention_kernel<T, E8, HD, 2><<<p.workgroups, 64 * WAVES, 0, st>>>(a, p, scratch, items);
    else if constexpr (HD == 256) paged_attention_kernel<T, E8, HD, 4><<<p.workgroups, 64 * WAVES, 0, st>>>(a, p, scratch, items);
    paged_attention_join_kernel<T, E8, HD><<<dim3(p.tiles * a.cache.n_kv_heads, a.rows.B), 256, 0, st>>>(a, p, scratch, items);
}

template <typename T, bool E8>
void launch_hd(const Attend &a, const Split &p, float *scratch, hipStream_t st) {
    if (a.cache.head_dim == 64) launch<T, E8, 64>(a, p, scratch, st);
    else if (a.cache.head_dim == 128) launch<T, E8, 128>(a, p, scratch, st);
    else launch<T, E8, 256>(a, p, scratch, st);
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
    if (!c || !rows || !cache || !attn || n_rows <= 0 || rows->B <= 0 || rows->max_new <= 0 || cache->n_kv_heads <= 0 ||
        attn->n_heads < cache->n_kv_heads)
        return 0;
    const long per_head = most_rows(n_rows, *rows, attn->n_heads / cache->n_kv_heads);
    if (prompt_takes(per_head, cache->head_dim))
        return prompt_scratch_floats(per_head, rows->B, cache->n_kv_heads, (long)cache->max_pages * cache->page_size, cache->head_dim,
                                     ctx_view(c).nCU) * sizeof(float);
    const Split p = split_of(per_head, cache->head_dim, ctx_view(c).nCU);
    return partial_floats(p, cache->head_dim) * sizeof(float) + (size_t)rows->B * p.tiles * cache->n_kv_heads * sizeof(Pieces);
}

int mrp_paged_attention(mrp_ctx *c, void *stream, long n_rows, const mrp_new_rows *rows, const mrp_paged_cache *cache,
                        const mrp_attn *attn, const void *q, long q_stride, void *out, float *lse, void *scratch, size_t scratch_bytes) {
    const char *what = "mrp_paged_attention";
    if (!c) return MRP_ERR_NULL;
    if (!rows || !cache || !attn) return ctx_fail(c, MRP_ERR_NULL, "%s: NULL pointer", what);
    CHECK(check_new_rows(c, what, n_rows, rows));
    CHECK(check_cache(c, what, cache, rows->B));
    if (attn->n_heads < 1 || attn->n_heads > 1024 || attn->n_heads % cache->n_kv_heads)
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %d heads over %d key heads", what, attn->n_heads, cache->n_kv_heads);
    if (n_rows * attn->n_heads > (1L << 28) || most_rows(n_rows, *rows, attn->n_heads / cache->n_kv_heads) > (1L << 22) ||
        (long)rows->B * cache->n_kv_heads > (1L << 22))
        return ctx_fail(c, MRP_ERR_SHAPE, "%s: %ld rows of %d heads, %d sequences of %d key heads are too many", what, n_rows, attn->n_heads,
                        rows->B, cache->n_kv_heads);
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
    Attend a = {*rows, *cache, *attn, (int)n_rows, attn->n_heads / cache->n_kv_heads, static_cast<const uint16_t *>(q), q_stride,
                      static_cast<uint16_t *>(out), lse, ctx_view(c).err_flag};
    if (attn->window > (long)cache->max_pages * cache->page_size) a.attn.window = 0;   // (wider than any sequence: none)
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (prompt_takes(most_rows(n_rows, *rows, a.G), cache->head_dim)) {
        const hipError_t e = launch_prompt_attention(a, static_cast<float *>(scratch), ctx_view(c).nCU, st);
        return e == hipSuccess ? MRP_OK : ctx_fail(c, MRP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    }
    const bool e8 = cache->dtype == MRP_DTYPE_E4M3;
    const Split p = split_of(most_rows(n_rows, *rows, a.G), cache->head_dim, ctx_view(c).nCU);
    float *const s = static_cast<float *>(scratch);
    if (attn->dtype == MRP_DTYPE_BF16) e8 ? launch_hd<BF16, true>(a, p, s, st) : launch_hd<BF16, false>(a, p, s, st);
    else e8 ? launch_hd<F16, true>(a, p, s, st) : launch_hd<F16, false>(a, p, s, st);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MRP_OK : ctx_fail(c, MRP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // extern "C"
