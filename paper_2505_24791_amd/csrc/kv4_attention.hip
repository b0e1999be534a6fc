// Attention of new tokens over a key/value cache held in 4 bits.
//
//   o_r = sum_t p_rt v_t / sum_t p_rt,   p_rt = exp(scale q_r . k_t - m_r),   over the keys t that row r sees
//
// One pass over the cache with the running maximum and sum of the softmax.  A key or value is a 4-bit float times a power of two and
// converts exactly to 16 bits, so the products on the matrix unit have exact right operands; only the probabilities are rounded, to the
// type of the rows (float32 rows: every left operand as three bfloat16 pieces, which hold its 24 bits, on the same instruction).
#include "kv4.h"

#include <type_traits>

namespace sjd {

namespace {

template <typename T> struct Op { typedef T t; static constexpr int pieces = 1; };
template <> struct Op<float> { typedef bf16 t; static constexpr int pieces = 3; };

typedef uint32_t u32;

// two values (a byte) of w with the scale s
template <typename HT, int SEL> __device__ __forceinline__ void decode2(u32 w, float s, HT &a, HT &b) {
    if constexpr (__is_same(HT, f16)) {
        const auto x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, SEL);
        a = x[0]; b = x[1];
    } else {
        const auto x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL);
        a = x[0]; b = x[1];
    }
}
template <typename HT> __device__ __forceinline__ void decode8(u32 w, float s, typename Half16<HT>::v8 &x) {
    HT a, b;
    decode2<HT, 0>(w, s, a, b); x[0] = a; x[1] = b;
    decode2<HT, 1>(w, s, a, b); x[2] = a; x[3] = b;
    decode2<HT, 2>(w, s, a, b); x[4] = a; x[5] = b;
    decode2<HT, 3>(w, s, a, b); x[6] = a; x[7] = b;
}
__device__ __forceinline__ float pow2_byte(u32 w, int i) { return __uint_as_float(((w >> (8 * i)) & 255u) << 23); }

// x as a sum of `n` values of the operand type, the largest first
template <typename T, int N> __device__ __forceinline__ void split(float x, typename Op<T>::t (&p)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = from_f32<typename Op<T>::t>(x);
        x -= to_f32<typename Op<T>::t>(p[i]);
    }
}

// Over the four lanes of a row (16 lanes apart): a swap of a register with itself leaves, in its two results, what the lanes of a pair hold.
template <typename F> __device__ __forceinline__ float over_row(float v, F f) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_max(float v) { return over_row(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ __forceinline__ float row_sum(float v) { return over_row(v, [](float x, float y) { return x + y; }); }

struct Seq { int row0, n, len, all; };      // first row, rows and keys of a sequence, within what the call allows; rows that it would have
__device__ __forceinline__ Seq sequence(const Kv4Attn &a, int b) {
    Seq s;
    if (a.q_start) {
        s.row0 = min(max(a.q_start[b], 0), a.n_rows);
        s.all = min(max(a.q_start[b + 1], s.row0), a.n_rows) - s.row0;
        s.n = min(s.all, a.max_q);
    } else {
        s.row0 = b * a.max_q;
        s.n = s.all = a.max_q;
    }
    s.len = min(min(max(a.kv_len[b], 0), a.max_kv), a.max_pages * kKv4Page);
    return s;
}
// keys first .. last of the i-th new token of a sequence (none: last < first)
__device__ __forceinline__ void seen(const Kv4Attn &a, const Seq &s, int i, int &first, int &last) {
    last = max((a.causal ? s.len - s.all + i : s.len - 1) - a.skip, -1);
    first = a.window ? max(0, last - a.window + 1) : 0;
}

// ------------------------------------------------------------------------------------------------
// 16 NT rows (new tokens times query heads of one key head) a workgroup, the pages of its piece of the sequence dealt to four
// waves, each with its own maximum and sums, which are joined at the end.  S^T = K Q^T, 16 tokens an instruction: a lane holds row lane % 16 and, of a subtile, tokens 4 (lane / 16) + 0..3, which is
// the right operand of O^T = V^T P^T as it stands, two subtiles to an instruction.
// Single tokens are bound by the cache's bytes: 16 sequences of 20000 to 65536 keys, 8 key heads of 128 (745 MB), 157 us a call with the join, 4.75 TB/s;
// 256 sequences of up to 1024 keys, 12 heads of 64 (108 MB), 29 us, of which 20 are bytes and the rest the longest sequences' workgroups.  Chunks of new
// tokens are bound by the vector ALU (an exponential of 12 cycles a score, the conversion of the codes for every 32 rows): 8 of 500 rows over 4000 keys, 16
// heads of 64, 99 us, 620 TFLOP/s of the products that rows see; and by the uneven ends of ragged sequences: 8 of up to 500 rows over 500 to 4000 keys, 61
// us, 270 TFLOP/s.  Whole prompts of 1024 tokens, 32 of them: 16 heads of 64 191 us, 360 TFLOP/s; 32 heads on 8 of 128 638 us, 431.
// Registers hold what a page needs and nothing is shared through LDS before the end: pages converted once into LDS for four waves were no
// faster on such sequences.
constexpr int kRows = 16;
constexpr float kLag = 8.f;                       // base 2
// The reference m of a row lies `over` below the maximum that it was taken from, so that the largest probability of a wave is 2^over to 2^(over + kLag).
// Half: 2^15 still fits, and probabilities down to 2^-21 of the largest keep their 11 bits, those down to 2^-32 are there; with m at the maximum itself
// a wave lost every key 17.4 nats below its leading one, however many they are.  The other types have the exponents of float32.
template <typename HT> constexpr float kOver = __is_same(HT, f16) ? 7.f : 0.f;

// the new token of a row (rows are the query heads of a key head, token by token)
__device__ __forceinline__ int token_of(const Kv4Attn &a, int row) { return a.group_magic ? (int)__umulhi((uint32_t)row, a.group_magic) : row; }

struct Tile { int first_lo, last_lo, first_hi, last_hi; };      // what the tile's first and last row see
__device__ __forceinline__ Tile tile_range(const Kv4Attn &a, const Seq &s, int r0, int n_r) {
    Tile t;
    seen(a, s, token_of(a, r0), t.first_lo, t.last_lo);
    seen(a, s, token_of(a, min(r0 + a.tile, n_r) - 1), t.first_hi, t.last_hi);
    return t;
}

// A page as one lane holds it: per subtile of 16 tokens NG dwords of keys and NG of values, the scales of its key (one dword for the four
// subtiles and each of its groups), and the value scales dealt over the 16 lanes that need the same ones.
template <int NG> struct Page {
    static constexpr int KS = NG > 4 ? NG / 4 : 1, VS = NG > 4 ? NG / 4 : 1;
    u32 k[4][NG], v[4][NG], ks[KS], vs[VS];
};
template <int NG> __device__ __forceinline__ void load_dwords(u32 (&d)[NG], const uint8_t *p) {
    typedef u32 vec __attribute__((ext_vector_type(NG == 1 ? 2 : NG > 4 ? 4 : NG)));
    if constexpr (NG == 1) d[0] = *reinterpret_cast<const u32 *>(p);
    else {
        constexpr int W = NG > 4 ? 4 : NG;
#pragma unroll
        for (int i = 0; i < NG; i += W) {
            const vec x = *reinterpret_cast<const vec *>(p + 4 * i);
#pragma unroll
            for (int e = 0; e < W; ++e) d[i + e] = x[e];
        }
    }
}
template <int NG> __device__ __forceinline__ void load_keys(Page<NG> &p, const uint8_t *blk, int r, int j) {
    constexpr int DIM = 32 * NG;
#pragma unroll
    for (int i = 0; i < Page<NG>::KS; ++i) p.ks[i] = *reinterpret_cast<const u32 *>(blk + kv4_k_scale(DIM, r, j * NG / 4 + i));
#pragma unroll
    for (int t = 0; t < 4; ++t) load_dwords<NG>(p.k[t], blk + kv4_k_code(DIM, 16 * t + r, j * NG));
}
template <int NG> __device__ __forceinline__ void load_values(Page<NG> &p, const uint8_t *blk, int r, int j) {
    constexpr int DIM = 32 * NG;
#pragma unroll
    for (int i = 0; i < Page<NG>::VS; ++i)
        p.vs[i] = *reinterpret_cast<const u32 *>(blk + kv4_v_scale(DIM, 4 * j) + 4 * (min(r, 4 * NG - 1) + 16 * i));
#pragma unroll
    for (int t = 0; t < 4; ++t) load_dwords<NG>(p.v[t], blk + kv4_v_code(DIM, 16 * t + 4 * j, r));
}
// lane I of every 16
template <int I> __device__ __forceinline__ u32 row_bcast(u32 x) {
    return (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x150 + I, 0xf, 0xf, true);      // row_newbcast
}
template <int N, int I = 0, typename F> __device__ __forceinline__ void unroll(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unroll<N, I + 1>(f);
    }
}

template <typename T, int NG, int NT>
__global__ __launch_bounds__(256, sizeof(T) == 4 && NG > 4 ? 1 : sizeof(T) == 4 || NG > 4 || NT * NG > 4 ? 2 : NT == 1 && NG <= 2 ? 5 : 3) void kv4_attention_kernel(Kv4Attn a) {
    typedef typename Op<T>::t HT;
    typedef typename Half16<HT>::v8 v8;
    typedef T qv8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    constexpr int NP = Op<T>::pieces, DIM = 32 * NG;
    constexpr int RG = NG < 4 ? NG : 4, RDIM = 32 * RG, LD = RDIM + 4;      // groups joined at a time
    __shared__ __attribute__((aligned(16))) float acc[4][kRows * LD];
    __shared__ float ms[4][kRows], ls[4][kRows];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, j = lane >> 4;
    const int G = a.group;
    // pieces further back come last: only long sequences have them
    const int z = blockIdx.z + a.z0;
    const int h = blockIdx.x, b = blockIdx.y, part = a.n_tiles == 1 ? z : z / a.n_tiles, tile = z - part * a.n_tiles;
    const Seq sq = sequence(a, b);
    const int n_r = sq.n * G, r0 = tile * (kRows * NT);
    if (r0 >= n_r) return;
    const Tile tr = tile_range(a, sq, r0, n_r);
    const int lo = tr.first_lo, hi = tr.last_hi;
    const int p0 = max(lo / kKv4Page, part * a.split_pages);
    const int p1 = min(hi < lo ? 0 : hi / kKv4Page + 1, (part + 1) * a.split_pages);
    if (p0 >= p1 && a.n_splits > 1) return;
    int first[NT], last[NT];                      // what row r0 + 16 n + r sees
#pragma unroll
    for (int n = 0; n < NT; ++n) seen(a, sq, token_of(a, min(r0 + kRows * n + r, n_r - 1)), first[n], last[n]);

    // The wave's pages (every fourth of the piece): first those that every row sees whole, f0 .. f1 - 1, then the ones after and before.
    const int f0 = min(max((tr.first_hi + kKv4Page - 1) / kKv4Page, p0), p1), f1 = max(min((tr.last_lo + 1) / kKv4Page, p1), f0);
    auto mine = [&](int from) { return from + ((wave - (from - p0)) & 3); };           // the first of them from there on
    auto count = [&](int from, int to) { return max(0, (to - mine(from) + 3) / 4); };
    const int n_whole = count(f0, f1), n_after = count(f1, p1), n_pages = n_whole + n_after + count(p0, f0);
    auto page_at = [&](int i) {
        return i < n_whole ? mine(f0) + 4 * i : i < n_whole + n_after ? mine(f1) + 4 * (i - n_whole) : mine(p0) + 4 * (i - n_whole - n_after);
    };
    // the table's entry is fetched two pages ahead, the page one ahead
    const int32_t *table = a.table + b * a.table_stride;
    const uint8_t *base = a.cache.pages + (size_t)h * kv4_block_bytes(DIM);
    const size_t page_bytes = (size_t)a.cache.n_heads * kv4_block_bytes(DIM);
    auto entry = [&](int i) { return i < n_pages ? table[page_at(i)] : -1; };
    auto valid = [&](int id) { return id >= 0 && id < a.cache.n_pages; };
    // what comes next is requested always, from some page where there is none: the compiler counts the loads on their way
    auto block = [&](int id) { return base + (size_t)(valid(id) ? id : 0) * page_bytes; };
    int id = entry(0), id_next = entry(1);
    Page<NG> pg;
    load_keys<NG>(pg, block(id), r, j);
    load_values<NG>(pg, block(id), r, j);

    v8 qf[NT][NG][NP];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = min(r0 + kRows * n + r, n_r - 1), tok = token_of(a, row);
        const T *q = (const T *)a.q + (int64_t)(sq.row0 + tok) * a.q_stride + (int64_t)(h * G + row - tok * G) * DIM;
#pragma unroll
        for (int s = 0; s < NG; ++s) {
            const qv8 x = *reinterpret_cast<const qv8 *>(q + 8 * (j * NG + s));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                HT p[NP];
                if constexpr (NP == 1) p[0] = x[e];
                else split<T, NP>(x[e], p);
#pragma unroll
                for (int c = 0; c < NP; ++c) qf[n][s][c][e] = p[c];
            }
        }
    }
    f32x4v o[NT][NG][2];
    float m[NT], l[NT];                           // of the row (the reference, scaled, base 2); of the lane's tokens of the row
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int g = 0; g < NG; ++g) o[n][g][0] = o[n][g][1] = f32x4v{0.f, 0.f, 0.f, 0.f};
        m[n] = -INFINITY;
        l[n] = 0.f;
    }

    // One page: scores, then the keys of the next page are requested; softmax; values, then those of the next page.
    auto step = [&](auto masked_, int page) {
        constexpr bool MASKED = decltype(masked_)::value;
        const int t0 = page * kKv4Page;
        f32x4v sc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < 4; ++t) sc[n][t] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 4; t += 2)
#pragma unroll
            for (int s = 0; s < NG; ++s) {
#pragma unroll
                for (int u = t; u < t + 2; ++u) {
                    v8 kf;
                    decode8<HT>(pg.k[u][s], pow2_byte(pg.ks[s / 4], u), kf);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < NP; ++c) sc[n][u] = Mfma16<HT>::run(kf, qf[n][s][c], sc[n][u]);
                }
                __builtin_amdgcn_sched_barrier(0);      // or all conversions of the page are begun at once, in as many registers
            }
        load_keys<NG>(pg, block(id_next), r, j);
        float m_use[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = t0 + 16 * t + 4 * j + e;
                    if (MASKED) sc[n][t][e] = key >= first[n] && key <= last[n] ? sc[n][t][e] : -INFINITY;
                    mx = fmaxf(mx, sc[n][t][e]);
                }
            // The running maximum is only a reference: it moves when a score of some row is more than 2^kLag times over it, so that pages seldom
            // exchange anything between lanes or touch the sums.
            mx *= a.scale_log2;
            if (__builtin_amdgcn_ballot_w64(!(mx <= m[n] + (kLag + kOver<HT>))) != 0) {
                const float m_new = fmaxf(m[n], row_max(mx) - kOver<HT>);
                const float corr = __builtin_amdgcn_exp2f(m[n] - (m_new == -INFINITY ? 0.f : m_new));
                l[n] *= corr;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][g][c][e] *= corr;
                m[n] = m_new;
            }
            m_use[n] = m[n] == -INFINITY ? 0.f : m[n];
        }
        // value scales as floats, byte k of a dword in vf[i][k], still dealt over the lanes
        u32 sf[Page<NG>::VS][4];
        constexpr u32 E = 0x7f800000u;
#pragma unroll
        for (int i = 0; i < Page<NG>::VS; ++i) {
            sf[i][0] = (pg.vs[i] << 23) & E;
            sf[i][1] = (pg.vs[i] << 15) & E;
            sf[i][2] = (pg.vs[i] << 7) & E;
            sf[i][3] = (pg.vs[i] >> 1) & E;
        }
        bool nan_hidden = false;
        if (MASKED) {
            // what no row sees is nothing's, and may be anything; a NaN that some row sees must not reach the others as 0 * NaN
#pragma unroll
            for (int i = 0; i < Page<NG>::VS; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int B = 4 * (min(r, 4 * NG - 1) + 16 * i) + k, key = t0 + 16 * (B / (4 * NG)) + 4 * j + B / NG % 4;
                    const bool any = key >= lo && key <= hi, bad = sf[i][k] == E;
                    nan_hidden |= any && bad;
                    sf[i][k] = any && !bad ? sf[i][k] : 0u;
                }
        }
        unroll<2>([&](auto half_) {
            constexpr int t = 2 * decltype(half_)::value;
            v8 pf[NT][NP];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[n][t + e / 4][e % 4], a.scale_log2, -m_use[n]));
                    HT p[NP];
                    if constexpr (NP == 1) p[0] = from_f32<HT>(x);
                    else { split<T, NP>(x, p); l[n] += x; }
#pragma unroll
                    for (int c = 0; c < NP; ++c) pf[n][c][e] = p[c];
                }
                if constexpr (NP == 1) l[n] = Half16<HT>::add_all(pf[n][0], l[n]);
            }
            unroll<NG>([&](auto g_) {
                constexpr int g = decltype(g_)::value;
                v8 vf[2];
                unroll<8>([&](auto e_) {
                    constexpr int e = decltype(e_)::value;
                    constexpr int at = (e % 4) * NG + g;                   // byte of the subtile's codes, and of its scales
                    constexpr int tt = t + e / 4, B = tt * 4 * NG + at;
                    const float s = __uint_as_float(row_bcast<(B / 4) % 16>(sf[B / 64][B % 4]));
                    HT x0, x1;
                    decode2<HT, at % 4>(pg.v[tt][at / 4], s, x0, x1);
                    vf[0][e] = x0;
                    vf[1][e] = x1;
                });
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < NP; ++c) {
                        o[n][g][0] = Mfma16<HT>::run(vf[0], pf[n][c], o[n][g][0]);
                        o[n][g][1] = Mfma16<HT>::run(vf[1], pf[n][c], o[n][g][1]);
                    }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        load_values<NG>(pg, block(id_next), r, j);
        if (MASKED && __builtin_amdgcn_ballot_w64(nan_hidden) != 0) {
            const uint8_t *blk = block(id);
            for (int off = 0; off < kKv4Page; ++off)
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if (t0 + off >= first[n] && t0 + off <= last[n] && blk[kv4_v_scale(DIM, off) + g] == 255)
                            o[n][g][0] = o[n][g][1] = f32x4v{NAN, NAN, NAN, NAN};
        }
    };
    auto walk = [&](auto masked_, int from, int to) {
        for (int i = from; i < to; ++i) {
            const int id_after = entry(i + 2);
            if (valid(id)) {
                step(masked_, page_at(i));
            } else {                              // not seen, and the next page not on its way yet
                load_keys<NG>(pg, block(id_next), r, j);
                load_values<NG>(pg, block(id_next), r, j);
            }
            id = id_next;
            id_next = id_after;
        }
    };
    walk(std::false_type{}, 0, n_whole);
    walk(std::true_type{}, n_whole, n_pages);

    // the four waves' sums, 16 rows and RG groups at a time
    const int orow = threadIdx.x >> 4, oc = threadIdx.x & 15;      // 16 threads a row, RDIM / 16 channels each
    constexpr int PER = RDIM / 16;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int rn = r0 + kRows * n;
        if (rn >= n_r) break;
        if (n) __syncthreads();
        const float ln = row_sum(l[n]);
        if (j == 0) { ms[wave][r] = m[n]; ls[wave][r] = ln; }
        const bool live = rn + orow < n_r;
        const int tok = token_of(a, rn + orow), head = h * G + rn + orow - tok * G;
        const int64_t at = sq.row0 + tok;
#pragma unroll
        for (int g0 = 0; g0 < NG; g0 += RG) {
            if (g0) __syncthreads();
#pragma unroll
            for (int g = 0; g < RG; ++g) {
                float *d = &acc[wave][r * LD + 32 * g + 8 * j];
                const f32x4v x = o[n][g0 + g][0], y = o[n][g0 + g][1];
                *reinterpret_cast<f32x4 *>(d) = f32x4{x[0], y[0], x[1], y[1]};
                *reinterpret_cast<f32x4 *>(d + 4) = f32x4{x[2], y[2], x[3], y[3]};
            }
            __syncthreads();
            const float mj = fmaxf(fmaxf(ms[0][orow], ms[1][orow]), fmaxf(ms[2][orow], ms[3][orow]));
            const float mu = mj == -INFINITY ? 0.f : mj;
            float w[4], den = 0.f, sum[PER];
#pragma unroll
            for (int i = 0; i < 4; ++i) { w[i] = __builtin_amdgcn_exp2f(ms[i][orow] - mu); den = fmaf(w[i], ls[i][orow], den); }
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                sum[e] = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[e] = fmaf(w[i], acc[i][orow * LD + oc * PER + e], sum[e]);
            }
            if (!live) continue;
            if (a.n_splits == 1) {
                T *out = (T *)a.o + at * a.o_stride + (int64_t)head * DIM + 32 * g0 + oc * PER;
                const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
                for (int e = 0; e < PER; ++e) out[e] = from_f32<T>(den == 0.f ? 0.f : sum[e] * inv);
            } else {
                const int64_t piece = (at * a.n_heads + head) * a.n_splits + part;
                float *out = a.partial + piece * DIM + 32 * g0 + oc * PER;
#pragma unroll
                for (int e = 0; e < PER; ++e) out[e] = sum[e];
                if (g0 == 0 && oc == 0) { a.partial_ml[2 * piece] = mj; a.partial_ml[2 * piece + 1] = den; }
            }
        }
    }
}

// Joins the pieces of a row and head: 16 lanes, or four times 16 (WIDE) that take every fourth piece, so that a row is one or two rounds of
// requests (16 sequences of up to 16 pieces, 32 heads of 128: 6 us).
template <typename T, int NG, bool WIDE>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4Attn a) {
    constexpr int DIM = 32 * NG, PER = 2 * NG, AHEAD = NG > 4 ? 4 : 8, LANES = WIDE ? 64 : 16, WAYS = LANES / 16;
    typedef T tv __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
    typedef float fv __attribute__((ext_vector_type(PER), aligned(8)));
    const int G = a.group, c = threadIdx.x & 15, way = (threadIdx.x & (LANES - 1)) >> 4;
    const int64_t id = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int head = (int)(id % a.n_heads), i = (int)(id / a.n_heads % a.max_q);
    const int64_t b = id / a.n_heads / a.max_q;
    if (b >= a.n_seqs) return;
    const Seq sq = sequence(a, (int)b);
    if (i >= sq.n) return;
    const Tile tr = tile_range(a, sq, (i * G + head % G) / a.tile * a.tile, sq.n * G);
    const int lo = tr.first_lo, hi = tr.last_hi;
    const int s0 = lo / kKv4Page / a.split_pages, s1 = hi < lo ? s0 : hi / kKv4Page / a.split_pages + 1;      // the pieces that have been written
    const int64_t at = sq.row0 + i, piece0 = (at * a.n_heads + head) * a.n_splits;
    const float *ml = a.partial_ml + 2 * piece0, *p = a.partial + piece0 * DIM + c * PER;
    float m = -INFINITY;
    for (int s = s0 + (threadIdx.x & (LANES - 1)); s < s1; s += LANES) m = fmaxf(m, ml[2 * s]);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, LANES));
    const float mu = m == -INFINITY ? 0.f : m;
    float den = 0.f, sum[PER] = {};
    for (int s = s0 + way; s < s1; s += WAYS * AHEAD) {
        fv x[AHEAD];
        float w[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int su = s + u * WAYS, at_u = min(su, s1 - 1);
            x[u] = *reinterpret_cast<const fv *>(p + (int64_t)at_u * DIM);
            w[u] = __builtin_amdgcn_exp2f(ml[2 * at_u] - mu);
            if (su < s1) den = fmaf(w[u], ml[2 * at_u + 1], den);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s + u * WAYS < s1)
#pragma unroll
                for (int e = 0; e < PER; ++e) sum[e] = fmaf(w[u], x[u][e], sum[e]);
    }
    if constexpr (WIDE) {
        den = row_sum(den);
#pragma unroll
        for (int e = 0; e < PER; ++e) sum[e] = row_sum(sum[e]);
        if (way) return;
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    tv out;
#pragma unroll
    for (int e = 0; e < PER; ++e) out[e] = from_f32<T>(den == 0.f ? 0.f : sum[e] * inv);
    *reinterpret_cast<tv *>((T *)a.o + at * a.o_stride + (int64_t)head * DIM + c * PER) = out;
}

}  // namespace

constexpr int kGridYZ = 65535;                    // workgroups of a grid's second and third dimension

bool kv4_attention_plan(Kv4Attn &a, bool is_f32) {
    a.group = a.n_heads / a.cache.n_heads;
    a.group_magic = a.group > 1 ? (uint32_t)(((1ull << 32) + a.group - 1) / a.group) : 0u;
    const int64_t rows = (int64_t)a.max_q * a.group;
    const int pages = (a.max_kv + kKv4Page - 1) / kKv4Page;
    // 32 rows a workgroup share the conversions of a page (8 sequences of 4000 keys, 8 key heads of 64, 1200 rows each: 156 us with 16 rows, 129
    // with 32), but a short launch is over sooner on 16 (one sequence of 1000 keys, 24 rows: 9.0 us, 10.4 with 32).  Registers hold two
    // such tiles up to heads of 128.
    const int64_t n_pairs = (int64_t)a.n_seqs * a.cache.n_heads;
    a.tile = rows > kRows && !is_f32 && a.cache.dim <= 128 && n_pairs * pages >= 256 ? 2 * kRows : kRows;
    // Pieces: workgroups for the chip a few times over (16 sequences of 20000 to 65536 keys, 8 key heads of 128: 1024 workgroups 171 us, 2048 148,
    // 4096 152 and a longer join); fewer of 32 rows, whose sums take longer to write and join than a few pages to read.
    a.n_tiles = (int)((rows + a.tile - 1) / a.tile);
    // workgroups with rows: sequences share n_rows between them
    const int64_t shared = (int64_t)a.cache.n_heads * ((int64_t)a.n_rows * a.group / a.tile + a.n_seqs), have = n_pairs * a.n_tiles < shared ? n_pairs * a.n_tiles : shared;
    const int64_t aim = a.tile == kRows ? 2048 : 1024;
    int64_t want = have ? (aim + have - 1) / have : 1;
    want = want < 1 ? 1 : want;
    int per = (int)((pages + want - 1) / want);
    per = (per + 3) / 4 * 4;                      // a page for each wave
    a.split_pages = per < 4 ? 4 : per;
    a.n_splits = (pages + a.split_pages - 1) / a.split_pages;
    if (a.n_splits < 1) a.n_splits = 1;
    // the grid's second dimension, and rows for which group_magic is exact
    return a.n_seqs <= kGridYZ && rows * a.group < (int64_t)1 << 31 && (int64_t)a.n_seqs * a.n_heads * a.max_q <= INT32_MAX;
}

size_t kv4_attention_workspace(const Kv4Attn &a) {
    return a.n_splits > 1 ? (size_t)a.n_rows * a.n_heads * a.n_splits * (a.cache.dim + 2) * sizeof(float) : 0;
}

template <typename T> void launch_tiles(const Kv4Attn &a, int n, hipStream_t s) {
    const dim3 grid(a.cache.n_heads, a.n_seqs, n), block(256);
    const int nt = a.tile / kRows;
#define SJD_KV4_ATTEND(NG, NT) hipLaunchKernelGGL((kv4_attention_kernel<T, NG, NT>), grid, block, 0, s, a)
    if constexpr (sizeof(T) == 4) {
        switch (a.cache.dim / 32) {
            case 1: SJD_KV4_ATTEND(1, 1); break;
            case 2: SJD_KV4_ATTEND(2, 1); break;
            case 4: SJD_KV4_ATTEND(4, 1); break;
            default: SJD_KV4_ATTEND(8, 1); break;
        }
    } else {
        switch (a.cache.dim / 32 * 8 + nt) {
            case 8 + 1: SJD_KV4_ATTEND(1, 1); break;
            case 8 + 2: SJD_KV4_ATTEND(1, 2); break;
            case 16 + 1: SJD_KV4_ATTEND(2, 1); break;
            case 16 + 2: SJD_KV4_ATTEND(2, 2); break;
            case 32 + 1: SJD_KV4_ATTEND(4, 1); break;
            case 32 + 2: SJD_KV4_ATTEND(4, 2); break;
            default: SJD_KV4_ATTEND(8, 1); break;
        }
    }
#undef SJD_KV4_ATTEND
}

template <typename T> void launch_kv4_attention(const Kv4Attn &a, hipStream_t s) {
    if (a.n_rows <= 0 || a.n_seqs <= 0 || a.n_tiles <= 0) return;
    const dim3 block(256);
    const int all = a.n_tiles * a.n_splits;
    Kv4Attn part = a;
    for (part.z0 = 0; part.z0 < all; part.z0 += kGridYZ) launch_tiles<T>(part, all - part.z0 < kGridYZ ? all - part.z0 : kGridYZ, s);
    if (a.n_splits > 1) {
        const int64_t rows = (int64_t)a.n_seqs * a.n_heads * a.max_q;
        const bool wide = a.n_splits > 8;         // one round of requests for 16 lanes
        const dim3 joins((unsigned)((rows + (wide ? 3 : 15)) / (wide ? 4 : 16)));
#define SJD_KV4_JOIN(NG)                                                                       \
    if (wide) hipLaunchKernelGGL((kv4_join_kernel<T, NG, true>), joins, block, 0, s, a);      \
    else hipLaunchKernelGGL((kv4_join_kernel<T, NG, false>), joins, block, 0, s, a)
        switch (a.cache.dim / 32) {
            case 1: SJD_KV4_JOIN(1); break;
            case 2: SJD_KV4_JOIN(2); break;
            case 4: SJD_KV4_JOIN(4); break;
            default: SJD_KV4_JOIN(8); break;
        }
#undef SJD_KV4_JOIN
    }
}
template void launch_kv4_attention<float>(const Kv4Attn &, hipStream_t);
template void launch_kv4_attention<bf16>(const Kv4Attn &, hipStream_t);
template void launch_kv4_attention<f16>(const Kv4Attn &, hipStream_t);

}  // namespace sjd
