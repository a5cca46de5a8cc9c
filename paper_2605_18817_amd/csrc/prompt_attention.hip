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
// their lanes.  Values are turned on their way into shared memory: entry d of all keys in row d / 2, the odd entries' rows behind the
// even ones', so that a lane ends up with neighbouring entries of its output row.
//
// Two prompts of 4096 and 3565 rows behind 3987 and 2190 positions, 32 heads of 128 over 8: 637 GFLOP in 733 us, 870 TFLOP/s.  A tile costs a
// wave 1024 cycles of the matrix core and about as many of the vector unit, 2800 in all for each of the two waves of a SIMD: within
// a wave they follow each other.  256 rows a workgroup rather than 128: 749 against 826 us, whose tiles are fetched and turned twice as often.
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

template <bool B>
struct Odd {
    static constexpr bool value = B;
};
using Even = Odd<false>;

struct Cut {
    int tiles;       // row tiles that a sequence can have
    int pieces;      // parts of a row tile's positions, at most; joined by a second kernel where there are more than one
    int slots;       // pieces that the whole batch is cut into, about
};

typedef const __attribute__((address_space(1))) void *gas_ptr;
typedef __attribute__((address_space(3))) void *las_ptr;

// Row of key x (0 .. 31) of a tile's half in shared memory, and the key of a row
__device__ __forceinline__ int key_row(int x) {
    const int i = 8 * (x >> 4) + (x & 7), h = (x >> 3) & 1;
    return 8 * (i >> 2) + 4 * h + (i & 3);
}

__device__ __forceinline__ int row_key(int y) {
    const int i = 4 * (y >> 3) + (y & 3), h = (y >> 2) & 1;
    return 16 * (i >> 3) + 8 * h + (i & 7);
}

// Partial results: per row tile and piece ROWS x (HD sums), then ROWS x (reference, sum of weights); behind them the pieces' size
__host__ __device__ inline size_t pieces_floats(int B, const Cut &P, int n_kv_heads, int rows, int HD) {
    return (size_t)B * P.tiles * n_kv_heads * P.pieces * rows * (HD + 2);
}
__device__ __forceinline__ int *size_place(const Attend &A, const Cut &P, float *scratch, int rows, int HD) {
    return reinterpret_cast<int *>(scratch + pieces_floats(A.rows.B, P, A.cache.n_kv_heads, rows, HD));
}

// Where the positions of 64 rows are cut: into as many parts for each sequence (32 caches of up to 8000 positions of 8 bits: 95 us; cut as
// below 117 to 126, whose few longer parts come in rounds)
__device__ __forceinline__ int even_size(int steps, int pieces) {
    const int size = (steps + pieces - 1) / pieces;
    return size < 1 ? 1 : size;
}

// Where the positions of more rows are cut: every so many tiles of them, the same for the whole batch, so that its pieces are about as
// many as find a place on the device, and none has to take longer than the others.  Worked out by all threads of a workgroup.
template <int THREADS>
__device__ __forceinline__ int piece_size(const Attend &A, const Cut &P, int rows, long cap) {
    __shared__ long totals[THREADS / 64];
    __shared__ int longest[THREADS / 64];
    long total = 0;
    int most = 0;
    for (int i = threadIdx.x; i < A.rows.B; i += THREADS) {
        const SeqRows s = seq_rows(A.rows, A.n_rows, cap, i);
        if (s.n == 0) continue;
        const int steps = steps_of<KT>(A.attn, s.len - s.n, s.len - 1, s.len).steps;
        total += (long)steps * ((s.n * A.G + rows - 1) / rows);
        most = most > steps ? most : steps;
    }
    for (int off = 32; off > 0; off >>= 1) {
        total += __shfl_xor(total, off);
        const int other = __shfl_xor(most, off);
        most = most > other ? most : other;
    }
    if ((threadIdx.x & 63) == 0) {
        totals[threadIdx.x >> 6] = total;
        longest[threadIdx.x >> 6] = most;
    }
    __syncthreads();
    total = 0;
    most = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        total += totals[w];
        most = most > longest[w] ? most : longest[w];
    }
    const long even = (total * A.cache.n_kv_heads + P.slots - 1) / P.slots, least = (most + P.pieces - 1) / P.pieces;
    const long size = even > least ? even : least;
    return size < 4 ? 4 : (int)size;
}

// x, hidden from what moves constant work out of loops
__device__ __forceinline__ int anew(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A load of W bytes
template <int W>
__device__ __forceinline__ uint32_t load_part(const char *p) {
    if constexpr (W == 4) return *reinterpret_cast<const uint32_t *>(p);
    else return *reinterpret_cast<const uint16_t *>(p);
}

// Orders the N products and the N reads of their operands above: reads four products ahead
template <int N>
__device__ __forceinline__ void four_ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < N - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
}

// NW waves; KH: the keys of a tile are halved between two waves with the same rows (2) or not (1)
template <typename T, bool E8, int HD, int NW, int KH>
__global__ __launch_bounds__(64 * NW, 2) void prompt_attention_kernel(const Attend A, const Cut P, float *scratch) {
    constexpr int ES = E8 ? 1 : 2, THREADS = 64 * NW, ROWS = 32 * NW / KH;
    constexpr int NT = 2 / KH;                    // halves of a tile that a wave takes
    constexpr int NC = HD / 16;                   // contraction steps of a score
    constexpr int ND = HD / 32;                   // tiles of 32 entries of the output
    constexpr int KROW = HD * 2;                  // bytes of a key's row in shared memory: piece x of row y lies in place x ^ y % KS,
    constexpr int KS = KROW / 16;                 // which spreads a piece of eight rows over the banks
    constexpr int VROW = KT * 2 + 16;             // bytes of an entry's: 16 more spread the rows
    constexpr int KP = HD * ES / 16;              // 16-byte pieces of a key in the cache
    constexpr int KN = KT * KP < THREADS ? 1 : KT * KP / THREADS;   // of them for a thread
    constexpr bool K_ALL = KT * KP >= THREADS;    // ... for every thread
    constexpr int DW = E8 ? 4 : 2;                // entries of a value that a thread takes
    constexpr int VL = HD / DW;                   // threads on a value
    constexpr int VK = KT * VL / THREADS;         // keys of a thread
    constexpr bool EARLY = KH == 2;
    static_assert(VK >= 2 && VK <= 16, "a thread's share");
    // (two variables, and the loop takes the tiles in pairs: what is on its way into one is then seen not to touch the other)
    __shared__ __align__(16) char ks_even[KT * KROW], ks_odd[KT * KROW];
    __shared__ __align__(16) char vs_even[HD * VROW], vs_odd[HD * VROW];
    __shared__ __align__(16) long places[4][KT];  // where the positions of four tiles lie, in bytes (0 where a page is not there)
    __shared__ uint32_t there[4][2];
    __shared__ int odd[4];                        // the tile has values that are not finite where only some rows see them

    const mrp_paged_cache &C = A.cache;
    const long cap = (long)C.max_pages * C.page_size;
    if (blockIdx.x == 0 && blockIdx.y == 0) check_rows(A.rows, A.n_rows, cap, A.err_flag, THREADS);
    // Key heads side by side: with eight of them, an XCD's L2 serves one, and one sequence at a time (two of 8083 and 5755 positions
    // side by side: 837 us instead of 723).  The last rows, which have the most to do, come first.
    const int kvh = blockIdx.x % C.n_kv_heads, rest = blockIdx.x / C.n_kv_heads, b = blockIdx.y, G = A.G;
    const SeqRows s = seq_rows(A.rows, A.n_rows, cap, b);
    const int nr = s.n * G, tiles = (nr + ROWS - 1) / ROWS;
    const int piece = rest % P.pieces, tile = tiles - 1 - rest / P.pieces;
    int size = 0x7fffffff;
    if (KH == 1 && P.pieces > 1) {
        size = piece_size<THREADS>(A, P, ROWS, cap);
        if (blockIdx.x == 0 && b == 0 && threadIdx.x == 0) *size_place(A, P, scratch, ROWS, HD) = size;   // (for the join)
    }
    if (tile < 0) return;
    const int row0 = tile * ROWS, last = row0 + ROWS < nr ? row0 + ROWS - 1 : nr - 1;
    const Steps st = steps_of<KT>(A.attn, s.len - s.n + row0 / G, s.len - s.n + last / G, s.len);
    if (KH == 2) size = even_size(st.steps, P.pieces);
    const bool pieces = st.steps > size;          // more than one
    const int begin = piece ? (int)((long)piece * size < st.steps ? piece * size : st.steps) : 0;
    const int n = (st.steps - begin < size ? st.steps - begin : size);
    if (piece && n == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r32 = lane & 31, h = lane >> 5;
    const int part = wave % (NW / KH), half = wave / (NW / KH);   // of the rows, and of a tile's keys

    // the row's position and operand (lanes past the last row take it again and store nothing)
    const int my = row0 + 32 * part + r32, r = my < nr ? my : nr - 1;
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
    // The first wave looks up the places of the piece's tile i: it asks for the page numbers a turn before it needs them
    auto ask = [&](int i) {
        const int j = key_of(begin + i) + (anew(threadIdx.x) & 63);
        return wave == 0 && any_sees(st, sink, j) ? table[j / C.page_size] : -1;
    };
    auto look_up = [&](int i, int page) {
        const int lane = anew(threadIdx.x) & 63, at = i & 3;
        if (wave == 0) {
            const int j = key_of(begin + i) + lane;
            const bool ok = page >= 0 && page < C.n_pages;
            if (!ok && any_sees(st, sink, j)) atomicOr(A.err_flag, ERR_PAGE);
            places[at][lane] = ok ? ((long)page * C.page_size + j % C.page_size) * pitch : 0;
            const unsigned long long all = __ballot(ok);
            if (lane == 0) {
                there[at][0] = (uint32_t)all;
                there[at][1] = (uint32_t)(all >> 32);
                odd[at] = 0;
            }
        }
    };
    int key_info[KN];                             // of a thread's pieces: where the place of their key is, and which part they are
#pragma unroll
    for (int n = 0; n < KN; ++n) {
        const int x = (n * NW + wave) * 64 + lane, y = x / KS;
        key_info[n] = 8 * ((y & 32) + row_key(y & 31)) | 16 * ((x % KS) ^ (y & (KS - 1))) << 16;
    }
    uint4 kreg[KN];                               // (8 bits: keys are widened on their way; else they go to shared memory directly)
    uint32_t vreg[VK];
    // (a thread's values: entries DW vd .., vd = tid % VL, of keys VK vg .., vg = tid / VL)
    // (what follows from a thread's number is worked out for each tile: kept, it would take the registers that the tile needs)
    auto request_direct = [&](int i, auto odd_tile) {
        if constexpr (!E8) {
            char *const ks = decltype(odd_tile)::value ? ks_odd : ks_even;
#pragma unroll
            for (int n = 0; n < KN; ++n) {        // 64 pieces of a wave lie side by side
                const int first = (n * NW + wave) * 64;
                const long place = *reinterpret_cast<const long *>(reinterpret_cast<const char *>(places[i & 3]) + (key_info[n] & 0xffff));
                __builtin_amdgcn_global_load_lds((gas_ptr)(kb + (key_info[n] >> 16) + place), (las_ptr)(ks + 16 * first), 16, 0, 0);
            }
            asm volatile("" ::: "memory");        // (what is asked for after it stays after it: the waits count)
        }
    };
    auto request = [&](int i) {
        const int tid = anew(threadIdx.x), vd = tid % VL, vg = tid / VL, at = i & 3;
        if constexpr (E8) {
#pragma unroll
            for (int n = 0; n < KN && (K_ALL || tid < KT * KP); ++n) {
                const int key = (tid + n * THREADS) / KP, part = (tid + n * THREADS) % KP;
                kreg[n] = *reinterpret_cast<const uint4 *>(kb + 16 * part + places[at][key]);
            }
        }
        const char *const vp = vb + DW * ES * vd;
#pragma unroll
        for (int n = 0; n < VK; ++n) vreg[n] = load_part<DW * ES>(vp + places[at][VK * vg + n]);
    };
    auto put = [&](int i, auto odd_tile) {
        const int tid = anew(threadIdx.x), vd = tid % VL, vg = tid / VL, u = begin + i, at = i & 3;
        char *const ks = decltype(odd_tile)::value ? ks_odd : ks_even, *const vs = decltype(odd_tile)::value ? vs_odd : vs_even;
        if constexpr (E8) {
#pragma unroll
            for (int n = 0; n < KN && (K_ALL || tid < KT * KP); ++n) {
                const int key = (tid + n * THREADS) / KP, part = (tid + n * THREADS) % KP, y = (key & 32) + key_row(key & 31);
                char *to = ks + y * KROW;
                uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
                widen(T{}, kreg[n].x, a0, a1);
                widen(T{}, kreg[n].y, a2, a3);
                widen(T{}, kreg[n].z, b0, b1);
                widen(T{}, kreg[n].w, b2, b3);
                *reinterpret_cast<uint4 *>(to + 16 * ((2 * part) ^ (y & (KS - 1)))) = make_uint4(a0, a1, a2, a3);
                *reinterpret_cast<uint4 *>(to + 16 * ((2 * part + 1) ^ (y & (KS - 1)))) = make_uint4(b0, b1, b2, b3);
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
            // values that no row sees are cleared; the tile is marked where others are not finite
            bool bad = false;
#pragma unroll
            for (int n = 0; n < VK; ++n) {
                const int k = VK * vg + n, j = key0 + k;
                const bool any = j < st.high && (j >= st.low || j < sink) && (((k & 32 ? th1 : th0) >> (k & 31)) & 1u);
#pragma unroll
                for (int i = 0; i < DW / 2; ++i) {
                    const uint32_t v = any ? w[n][i] : 0u;
                    bad |= not_finite(T{}, v);
                    w[n][i] = v;
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
            char *to = vs + ((d & 1) * (HD / 2) + (d >> 1)) * VROW + 2 * VK * vg;
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

    auto compute = [&](int i, auto odd_tile, auto after_scores, auto between) {
        const int lane = anew(threadIdx.x) & 63, r32 = lane & 31, h = lane >> 5, u = begin + i, at = i & 3;
        char *const ks = decltype(odd_tile)::value ? ks_odd : ks_even, *const vs = decltype(odd_tile)::value ? vs_odd : vs_even;
        const int key0 = key_of(u);
        const uint32_t th0 = there[at][0], th1 = there[at][1];
        f32x16 sc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int half_key = 32 * (KH == 2 ? half : t);
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[t][i] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const u32x4 a = *reinterpret_cast<const u32x4 *>(ks + (half_key + r32) * KROW + ((32 * c) ^ (16 * (h ^ (r32 & (KS - 1))))));
                sc[t] = mfma32(T{}, a, qf[c], sc[t]);
            }
        }
        four_ahead<NT * NC>();
        after_scores();
        const bool partial = is_partial(key0, th0, th1);
        float mx = LOWEST;
        if (partial) {
            uint32_t any = 0;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int tt = KH == 2 ? half : t;
                const uint32_t all = seen_bits(pos, key0 + 32 * tt, s.len, A.attn) & (tt ? th1 : th0), seen = all >> (8 * h);
                any |= all;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][i] = (seen >> (16 * (i >> 3) + (i & 7))) & 1u ? sc[t][i] : -INFINITY;
            }
            mx = any ? LOWEST : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16 * NT; ++i) mx = fmaxf(mx, sc[i >> 4][i & 15]);
        mx = max_halves(mx);
        // the sums are brought to a new reference where a weight would be more than 2^8 of the old one's unit
        float shift = Many<T>::SHIFT - reference(m, c2);
        if (__any(fmaf(mx, c2, shift) > 8.f + Many<T>::SHIFT || (m == -INFINITY && mx > m))) {
            const float top = fmaxf(m, mx);
            const float alpha = m == -INFINITY ? 0.f : exp2_((m - top) * c2);
            m = top;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] *= alpha;
            shift = Many<T>::SHIFT - reference(m, c2);
        }
        u32x4 p[2 * NT];                          // the weights of 16 keys each, rounded to 16 bits
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16 * NT; i += 2) {
            const float p0 = exp2_(fmaf(sc[i >> 4][i & 15], c2, shift)), p1 = exp2_(fmaf(sc[i >> 4][(i & 15) + 1], c2, shift));
            float x, y;
            sum += p0 + p1;
            p[i >> 3][(i & 7) >> 1] = pack2(T{}, p0, p1, x, y);
        }
        l += sum;
        between();
        if (partial && odd[at]) {
            // A weight of zero times a value that is not finite is not zero.  Such values leave the product; how many of them a row
            // sees in an entry is a product too, of ones, and makes the row's entry NaN
            u32x4 sees[2 * NT];
#pragma unroll
            for (int q = 0; q < 2 * NT; ++q) {
                const uint32_t seen = seen_bits(pos, key0 + 32 * (KH == 2 ? half : q >> 1), s.len, A.attn) >> (16 * (q & 1) + 8 * h);
#pragma unroll
                for (int j = 0; j < 4; ++j) sees[q][j] = ((seen >> (2 * j)) & 1u) * one_bits(T{}) + (((seen >> (2 * j + 1)) & 1u) * one_bits(T{}) << 16);
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                f32x16 count;
#pragma unroll
                for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll
                for (int q = 0; q < 2 * NT; ++q) {
                    u32x4 a = *reinterpret_cast<const u32x4 *>(vs + (32 * d + r32) * VROW + 32 * q + 64 * (KH == 2 ? half : 0) + 16 * h);
#pragma unroll
                    for (int j = 0; j < 4; ++j) a[j] = odd_halves(T{}, a[j]);
                    count = mfma32(T{}, a, sees[q], count);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] = count[i] > 0.f ? NAN : acc[d][i];
                __builtin_amdgcn_sched_barrier(0);
            }
            __syncthreads();                      // (all waves are here: the mark is the tile's)
            for (int x = tid; x < HD * (KT / 8); x += THREADS) {
                u32x4 *const v = reinterpret_cast<u32x4 *>(vs + (x / (KT / 8)) * VROW + 16 * (x % (KT / 8)));
                u32x4 a = *v;
#pragma unroll
                for (int j = 0; j < 4; ++j) a[j] = finite_halves(T{}, a[j]);
                *v = a;
            }
            __syncthreads();
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int q = 0; q < 2 * NT; ++q) {
                const u32x4 a = *reinterpret_cast<const u32x4 *>(vs + (32 * d + r32) * VROW + 32 * q + 64 * (KH == 2 ? half : 0) + 16 * h);
                acc[d] = mfma32(T{}, a, p[q], acc[d]);
            }
        four_ahead<2 * NT * ND>();
    };

    // three tiles are on their way: the places of the one after the next, keys and values of the next, and the one at work
    int page = -1;                                // of the tile that is looked up next
    if (n > 0) {
        const int page0 = ask(0), page1 = ask(1), page2 = ask(2), page3 = EARLY ? ask(3) : -1;
        look_up(0, page0);
        if (n > 1) look_up(1, page1);
        if (EARLY && n > 2) look_up(2, page2);
        page = EARLY ? page3 : page2;
        __syncthreads();
        request_direct(0, Even{});
        request(0);
        put(0, Even{});
        if (EARLY && n > 1) request(1);
    }
    // what goes to shared memory directly is there: nothing is on its way but what was asked for after it
    if (!E8 && EARLY && n > 1) __builtin_amdgcn_s_waitcnt(0x0F70 | (VK & 15) | (VK >> 4 << 14));
    else if (!E8) __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    auto step = [&](int i, auto odd_tile) {
        using Next = Odd<!decltype(odd_tile)::value>;
        // The next tile is asked for while the scores' products are under way, and its values are put in place ahead of the second
        // product: what a wave waits for is covered by what its matrix core does meanwhile.  EARLY: values (and keys of 8 bits) are
        // asked for a tile before that, since a tile's work is shorter than the memory takes; keys that go to shared memory
        // directly at the tile's begin.  The compiler waits for more than that: where the branches below join paths with different
        // numbers of requests it waits for all (16 bits: ahead of an even tile's first product, and of an odd tile's page numbers
        // and values; 8 bits: at the page number), so that less than a tile's work covers them
        if (EARLY && i + 1 < n) request_direct(i + 1, Next{});
        compute(i, odd_tile, [&] {
            if (EARLY) {
                if (i + 3 < n) look_up(i + 3, page);
                if (i + 4 < n) page = ask(i + 4);
            } else {
                if (i + 1 < n) {
                    request_direct(i + 1, Next{});
                    request(i + 1);
                }
                if (i + 2 < n) look_up(i + 2, page);
                if (i + 3 < n) page = ask(i + 3);
            }
        }, [&] {
            if (i + 1 < n) put(i + 1, Next{});
            if (EARLY && i + 2 < n) request(i + 2);
        });
        // the keys that go to shared memory directly are there: nothing is on its way but the VK values asked for after them
        if (!EARLY || i + 2 >= n) __builtin_amdgcn_s_waitcnt(0x0F70);
        else if (!E8) __builtin_amdgcn_s_waitcnt(0x0F70 | (VK & 15) | (VK >> 4 << 14));
        __syncthreads();
    };
    for (int i = 0; i < n; i += 2) {
        step(i, Even{});
        if (i + 1 < n) step(i + 1, Odd<true>{});
    }

    l += __shfl_xor(l, 32);
    if constexpr (KH == 2) {                      // the two waves of a row add up (the tiles' places are free)
        float *const mine = reinterpret_cast<float *>(part ? vs_odd : vs_even) + lane;
        if (half == 1) {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) mine[(16 * d + i) * 64] = acc[d][i];
            mine[16 * ND * 64] = m;
            mine[(16 * ND + 1) * 64] = l;
        }
        __syncthreads();
        if (half == 1) return;
        const float m1 = mine[16 * ND * 64], l1 = mine[(16 * ND + 1) * 64], top = fmaxf(m, m1);
        const float f0 = m == -INFINITY ? 0.f : exp2_((m - top) * c2), f1 = m1 == -INFINITY ? 0.f : exp2_((m1 - top) * c2);
        m = top;
        l = l * f0 + l1 * f1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = acc[d][i] * f0 + mine[(16 * d + i) * 64] * f1;
    }
    if (my >= nr) return;
    const bool empty = m == -INFINITY;
    const float v_scale = E8 && C.v_scale ? C.v_scale[kvh] : 1.f;
    if (pieces) {
        float *place = scratch + (((size_t)b * P.tiles + tile) * C.n_kv_heads + kvh) * P.pieces * ROWS * (HD + 2) + (size_t)piece * ROWS * (HD + 2);
        float *dst = place + (size_t)(32 * part + r32) * HD;
#pragma unroll
        for (int d = 0; d < ND / 2; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                float4 *to = reinterpret_cast<float4 *>(dst + 2 * (32 * d + 2 * i + 4 * h));
                to[0] = make_float4(acc[d][i], acc[d + ND / 2][i], acc[d][i + 1], acc[d + ND / 2][i + 1]);
                to[1] = make_float4(acc[d][i + 2], acc[d + ND / 2][i + 2], acc[d][i + 3], acc[d + ND / 2][i + 3]);
            }
        if (h == 0) *reinterpret_cast<float2 *>(place + (size_t)ROWS * HD + 2 * (32 * part + r32)) = make_float2(m, l);
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
    if (A.lse && h == 0) A.lse[at] = empty ? -INFINITY : m * c2 * 0.6931471805599453f + logf(l * (1.f / Many<T>::ONE));
}

// Adds up a row tile's pieces in the order of their positions: 16 threads a row, 16 rows a workgroup
template <typename T, bool E8, int HD, int ROWS>
__global__ __launch_bounds__(256) void prompt_join_kernel(const Attend A, const Cut P, const float *scratch) {
    constexpr int NE = HD / 16;
    const mrp_paged_cache &C = A.cache;
    const int per = ROWS / 16, b = blockIdx.y, slice = blockIdx.x % per, kvh = blockIdx.x / per % C.n_kv_heads, tile = blockIdx.x / per / C.n_kv_heads;
    const SeqRows s = seq_rows(A.rows, A.n_rows, (long)C.max_pages * C.page_size, b);
    const int rr = 16 * slice + (threadIdx.x >> 4), part = threadIdx.x & 15, r = tile * ROWS + rr;
    if (r >= s.n * A.G) return;
    const float c2 = A.attn.scale * 1.4426950408889634f * (E8 && C.k_scale ? C.k_scale[kvh] : 1.f);
    const int row0 = tile * ROWS;
    const int last = row0 + ROWS < s.n * A.G ? row0 + ROWS - 1 : s.n * A.G - 1;
    const int steps = steps_of<KT>(A.attn, s.len - s.n + row0 / A.G, s.len - s.n + last / A.G, s.len).steps;
    const int size = ROWS == 64 ? even_size(steps, P.pieces) : *size_place(A, P, const_cast<float *>(scratch), ROWS, HD);
    const int pieces = (steps + size - 1) / size;
    if (pieces <= 1) return;
    const float *place = scratch + (((size_t)b * P.tiles + tile) * C.n_kv_heads + kvh) * P.pieces * ROWS * (HD + 2);
    float mx = -INFINITY, sum = 0.f, o[NE];
    for (int q = 0; q < pieces; ++q) mx = fmaxf(mx, place[(size_t)q * ROWS * (HD + 2) + (size_t)ROWS * HD + 2 * rr]);
#pragma unroll
    for (int e = 0; e < NE; ++e) o[e] = 0.f;
    for (int q = 0; q < pieces; ++q) {
        const float *p = place + (size_t)q * ROWS * (HD + 2);
        const float2 ml = *reinterpret_cast<const float2 *>(p + (size_t)ROWS * HD + 2 * rr);
        const float f = ml.x == -INFINITY ? 0.f : exp2_((ml.x - mx) * c2);
        sum += f * ml.y;
        const float4 *src = reinterpret_cast<const float4 *>(p + (size_t)rr * HD + NE * part);
#pragma unroll
        for (int e = 0; e < NE; e += 4) {
            const float4 v = src[e / 4];
            o[e] += f * v.x; o[e + 1] += f * v.y; o[e + 2] += f * v.z; o[e + 3] += f * v.w;
        }
    }
    const int t = r / A.G;
    store_row<T, HD>(A, s.begin + t, kvh * A.G + r - t * A.G, part, mx == -INFINITY, mx * c2, Many<T>::ONE, sum, E8 && C.v_scale ? C.v_scale[kvh] : 1.f, o);
}

// Rows of a workgroup: 64 (four waves, keys halved between them), 128 (four waves) or 256 (eight)
int tile_rows(long rows) { return rows <= 64 ? 64 : (rows <= 128 ? 128 : 256); }

// Two workgroups of four waves find a place on a compute unit, one of eight.  Where the row tiles are few, their positions are cut into
// pieces of four tiles at least of the longest sequence that the table allows: for 64 rows into as many as give four workgroups a
// compute unit; for 128 into three rounds' worth, twice that for the longest (32 caches of up to 32767 positions, 32 rows of 4 heads
// each: one round 632 us, two 491, three 363; whole sequences 650); for 256 into one round's.
Cut cut_of(long rows, int B, int n_kv_heads, long positions, int nCU) {
    Cut c;
    const int per = tile_rows(rows);
    const long items = rows > 0 ? (rows + per - 1) / per * B * n_kv_heads : 0, longest = positions / (4 * KT);
    c.tiles = (int)((rows + per - 1) / per);
    c.slots = (per == 128 ? 6 : 1) * (nCU > 0 ? nCU : 1);
    long pieces = 1;
    if (items > 0) pieces = per == 64 ? 4 * (long)c.slots / items : (items < c.slots ? (2 * (long)c.slots + items - 1) / items : 1);
    if (pieces > longest) pieces = longest;
    c.pieces = pieces < 1 ? 1 : (int)pieces;
    return c;
}

template <typename T, bool E8, int HD, int NW, int KH>
void launch(const Attend &a, const Cut &c, float *scratch, hipStream_t st) {
    constexpr int ROWS = 32 * NW / KH;
    prompt_attention_kernel<T, E8, HD, NW, KH><<<dim3(c.tiles * a.cache.n_kv_heads * c.pieces, a.rows.B), 64 * NW, 0, st>>>(a, c, scratch);
    if (c.pieces > 1)
        prompt_join_kernel<T, E8, HD, ROWS><<<dim3(c.tiles * a.cache.n_kv_heads * (ROWS / 16), a.rows.B), 256, 0, st>>>(a, c, scratch);
}

template <typename T, bool E8, int HD>
void launch_form(const Attend &a, const Cut &c, int rows, float *scratch, hipStream_t st) {
    if (rows == 64) launch<T, E8, HD, 4, 2>(a, c, scratch, st);
    else if (rows == 128) launch<T, E8, HD, 4, 1>(a, c, scratch, st);
    else launch<T, E8, HD, 8, 1>(a, c, scratch, st);
}
template <typename T, bool E8>
void launch_hd(const Attend &a, const Cut &c, int rows, float *scratch, hipStream_t st) {
    if (a.cache.head_dim == 64) launch_form<T, E8, 64>(a, c, rows, scratch, st);
    else launch_form<T, E8, 128>(a, c, rows, scratch, st);
}

}  // namespace

// From 33 rows of a key head.  64 rows here / in paged_attention.hip's kernel (four waves, 16 rows each): 64 caches of up to 32767
// positions, bf16, 640 to 680 / 704 us; 32 of up to 8000, e4m3, 95 / 135.  32 rows there: 469, bf16.  (Heads of 256 stay there: their sums and
// queries would not fit a wave's registers here.)
bool prompt_takes(long rows, int head_dim) { return rows > 32 && head_dim <= 128; }

size_t prompt_scratch_floats(long rows, int B, int n_kv_heads, long positions, int head_dim, int nCU) {
    const Cut c = cut_of(rows, B, n_kv_heads, positions, nCU);
    return c.pieces > 1 ? pieces_floats(B, c, n_kv_heads, tile_rows(rows), head_dim) + 4 : 0;
}

hipError_t launch_prompt_attention(const Attend &a, float *scratch, int nCU, hipStream_t st) {
    const long rows = most_rows(a.n_rows, a.rows, a.G);
    const Cut c = cut_of(rows, a.rows.B, a.cache.n_kv_heads, (long)a.cache.max_pages * a.cache.page_size, nCU);
    const bool e8 = a.cache.dtype == MRP_DTYPE_E4M3;
    const int per = tile_rows(rows);
    if (a.attn.dtype == MRP_DTYPE_BF16) e8 ? launch_hd<BF16, true>(a, c, per, scratch, st) : launch_hd<BF16, false>(a, c, per, scratch, st);
    else e8 ? launch_hd<F16, true>(a, c, per, scratch, st) : launch_hd<F16, false>(a, c, per, scratch, st);
    return hipGetLastError();
}

}  // namespace mrp
