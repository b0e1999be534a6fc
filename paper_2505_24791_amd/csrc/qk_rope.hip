// Queries and keys normed for each head and rotated by their positions, and the cache of 4 bits written and read.
//
//   y = x / sqrt(mean x^2 + eps) * gain      or      (x - mean) / sqrt(var + eps) * gain + shift      (over the channels of a head)
//   (y_a, y_b) <- (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = position[axis of the pair] * frequency[pair]
//
// Everything between the load and the rounding (to float32, then to the rows' type) is float64: a value that lands next to a border of the 4-bit
// grid then goes to the same side in whatever order sums are taken (float32 sums in another order move one key in ten million to
// the next level, a third of its size), and angles of far positions keep their digits.  The vector unit does float64 at the rate
// of float32 here, and these kernels move bytes: each row is read once and written once.
#include "kv4.h"

namespace sjd {

namespace {

// A constant of the polynomials below, in scalar registers: the compiler would keep all of them in vector registers around the loops.
__device__ __forceinline__ double scalar(double x) {
    asm("" : "+s"(x));
    return x;
}

// cos and sin of p * f in float64.  The product of a 32-bit integer and a float32 needs 55 bits: taken as a sum of two doubles,
// and so are the turns p f / 2 pi, of which the whole ones go; the fraction is good to 2^-52 of a turn.  What is left after whole quarters, at
// most pi / 4, goes into the Taylor sums up to x^15 and x^16 (the next terms are below 5e-17).
__device__ __forceinline__ double2 unit(int32_t p, float f) {
#pragma clang fp contract(off)   // th below is the rounded product, also where it is subtracted from
    const double ah = (double)p * (double)f, al = fma((double)p, (double)f, -ah);
    const double ih = 0.15915494309189535, il = -9.839338337591243e-18;      // 1 / 2 pi
    const double th = ah * ih, tl = fma(ah, ih, -th) + fma(ah, il, al * ih);
    const double z = 4.0 * ((th - rint(th)) + tl), k = rint(z);
    const double x = (z - k) * 1.5707963267948966, xx = x * x;
    double s = scalar(-1.0 / 1307674368000), c = scalar(1.0 / 20922789888000);
    s = fma(s, xx, scalar(1.0 / 6227020800));
    c = fma(c, xx, scalar(-1.0 / 87178291200));
    s = fma(s, xx, scalar(-1.0 / 39916800));
    c = fma(c, xx, scalar(1.0 / 479001600));
    s = fma(s, xx, scalar(1.0 / 362880));
    c = fma(c, xx, scalar(-1.0 / 3628800));
    s = fma(s, xx, scalar(-1.0 / 5040));
    c = fma(c, xx, scalar(1.0 / 40320));
    s = fma(s, xx, scalar(1.0 / 120));
    c = fma(c, xx, scalar(-1.0 / 720));
    s = fma(s, xx, scalar(-1.0 / 6));
    c = fma(c, xx, scalar(1.0 / 24));
    s = fma(s * xx, x, x);
    c = fma(fma(c, xx, -0.5), xx, 1.0);
    const int quarter = (int)k;
    const double cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
    return {(quarter + 1) & 2 ? -cc : cc, quarter & 2 ? -ss : ss};
}

template <int CTRL> __device__ __forceinline__ double dpp_add(double v) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 x = __builtin_bit_cast(i32x2, v);
    const i32x2 y = {__builtin_amdgcn_update_dpp(0, x.x, CTRL, 0xf, 0xf, true), __builtin_amdgcn_update_dpp(0, x.y, CTRL, 0xf, 0xf, true)};
    return v + __builtin_bit_cast(double, y);
}
// over L neighbouring lanes: quads by permutation, then mirrors (what they mirror is the same in all lanes of a part)
template <int L> __device__ __forceinline__ double lanes_sum(double v) {
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    if constexpr (L >= 8) v = dpp_add<0x141>(v);
    if constexpr (L >= 16) v = dpp_add<0x140>(v);
    if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

__device__ __forceinline__ void turn(double &a, double &b, double2 u) {
    const double x = a;
    a = fma(x, u.x, -(b * u.y));
    b = fma(b, u.x, x * u.y);
}

// N values that start on a multiple of their own size
template <typename T, int N> struct Vec { typedef T v __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };

// Through float32, kept apart: in one step the compiler rounds float64 to 16 bits with thirty instructions of its own.
template <typename T> __device__ __forceinline__ typename Vec<T, 4>::v round4(const double *y) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef T t2 __attribute__((ext_vector_type(2)));
    const t2 a = __builtin_convertvector((f32x2{keep_f32((float)y[0]), keep_f32((float)y[1])}), t2);
    const t2 b = __builtin_convertvector((f32x2{keep_f32((float)y[2]), keep_f32((float)y[3])}), t2);
    return typename Vec<T, 4>::v{a[0], a[1], b[0], b[1]};
}

// Results go through the caches, however many: the call that reads them comes next.  Stores past the caches make a large call whose results nobody
// reads shorter (32768 tokens of 16 heads of 64 read back: 27 us, 41 through them) and a call with its reader longer, in a row of such pairs on inputs that
// change: those rows into the cache and attended over up to 1024 keys 251 us, 238 through the caches; 2 x 16 heads turned, and queries and keys read once, 109 and
// 98; read back, and keys and values read once, 75 and 69.  From 512 MB of results on, more than the last-level cache holds, the two are alike within 4%
// (385 and 384, 967 and 965, 295 and 304).
template <typename T, int N> __device__ __forceinline__ void store(T *p, typename Vec<T, N>::v v) { *reinterpret_cast<typename Vec<T, N>::v *>(p) = v; }

// Where a lane's two pieces of four channels begin: piece b holds the partners of piece a where the pairs are rot / 2 apart.
struct Pieces { int a, b; };
__device__ __forceinline__ Pieces pieces(int i, const QkOpts &o) {
    if (!o.adjacent && 8 * i < o.rot) return {4 * i, 4 * i + o.rot / 2};
    return {8 * i, 8 * i + 4};
}

// ---- 4 bits ----------------------------------------------------------------------------------

// The exponent byte of a group from the bits of its largest magnitude: the smallest power of two s with max <= 7 s, for 7 s rounds to
// 6 s with the error s that any value between 4 s and 6 s may have as well.  Bounded so that every held value and its half step
// exist in the rows' type.  255 where the group holds a NaN or an infinity.
template <typename T> __device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    constexpr int lo = sizeof(T) == 2 && __is_same(T, f16) ? 127 - 23 : 127 - 125, hi = __is_same(T, f16) ? 127 + 13 : 127 + 125;
    if (top >= 0x7f800000u) return 255;
    const int e = (int)((top + 0x1fffffu) >> 23) - 2;          // the carry: a mantissa above 1.75 takes the next power
    return (uint32_t)min(max(e, lo), hi);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight values in 4 bits each, round to nearest even, magnitudes over 6 become 6; byte 255: zeros (they read as NaN)
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], uint32_t byte) {
    if (byte == 255) return 0;
    const float s = scale_of(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// the largest of four neighbouring lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
}

// Where a token's block is, nullptr where the slot is outside the cache.
__device__ __forceinline__ uint8_t *block_of(const Kv4Cache &c, int32_t slot, int head) {
    if (slot < 0 || slot >= (int64_t)c.n_pages * kKv4Page) return nullptr;
    return c.pages + ((size_t)(slot / kKv4Page) * c.n_heads + head) * kv4_block_bytes(c.dim);
}

// Eight channels (the ch-th eight) of a token's key or value for one head; four neighbouring lanes hold a group.  b == nullptr: nothing is stored.
template <typename T> __device__ __forceinline__ void hold_key(uint8_t *b, int dim, int off, int ch, typename Vec<T, 8>::v r) {
    float x[8];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = to_f32<T>(r[e]); top = max(top, mag(x[e])); }
    const uint32_t sb = scale_byte<T>(quad_max(top));
    if (!b) return;
    *reinterpret_cast<uint32_t *>(b + kv4_k_code(dim, off, ch)) = encode8(x, sb);
    if (ch % 4 == 0) b[kv4_k_scale(dim, off, ch / 4)] = (uint8_t)sb;
}
template <typename T> __device__ __forceinline__ void hold_value(uint8_t *b, int dim, int off, int ch, typename Vec<T, 8>::v r) {
    float x[8];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = to_f32<T>(r[e]); top = max(top, mag(x[e])); }
    const uint32_t sb = scale_byte<T>(quad_max(top));
    if (!b) return;
    const uint32_t w = encode8(x, sb);
    uint8_t *d = b + kv4_v_code(dim, off, 4 * (ch % 4)) + ch / 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e * (dim / 8)] = (uint8_t)(w >> (8 * e));        // the next pair is 4 NG bytes on
    if (ch % 4 == 0) b[kv4_v_scale(dim, off) + ch / 4] = (uint8_t)sb;
}

// ---- kernels ---------------------------------------------------------------------------------

constexpr int kThreads = 256;

// A workgroup takes `per` rows, a power of two; L lanes (a group) take a head, eight channels each.  A group keeps its row and goes over every
// `step`-th head of it, so that addresses move by constants; the next head is requested under the present one's arithmetic.  cos and sin of every
// (row, pair) are made once for all heads, in LDS.  WRITE: rounded keys go to LDS instead of memory, and with the values from there into
// the cache.
// Bound by memory: 32768 rows of 2 x 16 heads of 64 (268 MB in and out) take 58 us a call in a row of calls, 4.6 TB/s, where a copy of 2 GiB runs at
// 5.0.  9945 rows of 40 heads of 128, three axes (204 MB): 55 us, beside float64 arithmetic of much the same length.  The 32768 rows into the cache
// (304 MB): 75 us.  Short calls are launch and one trip to memory: 32 rows 4.0 us.
struct RopeShape { int per, log_step; double per_dim; };

template <typename T, int L, bool WRITE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 4 : 5) void qk_rope_kernel(QkOpts o, QkRows r, Kv4Cache c, RopeShape sh) {
    typedef typename Vec<T, 4>::v v4;
    typedef typename Vec<T, 8>::v v8;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int pairs = o.rot / 2, quads = pairs / 4;
    double2 *cs = reinterpret_cast<double2 *>(smem);                                     // [per][4][quads]: a lane's four pairs apart, or neighbouring lanes meet in a bank
    float *affine = reinterpret_cast<float *>(cs + (size_t)sh.per * pairs);              // [4][dim] gains of q and k, shifts of q and k
    T *keys = reinterpret_cast<T *>(affine + 4 * r.dim);                                 // [per][n_kv][dim]
    const int tid = threadIdx.x, i = tid % L, group = tid / L, row0 = blockIdx.x * sh.per, rows = min(sh.per, r.n_rows - row0);
    const int step = 1 << sh.log_step, row = group >> sh.log_step, h0 = group & (step - 1);
    const int n_q = r.q ? r.n_heads : 0, n_k = r.k ? r.n_kv : 0;
    const int k0 = (unsigned)(h0 + (step - 1) * n_q) % (unsigned)step;                   // (h0 - n_q) mod step: groups that have no query head left begin with keys
    const Pieces p = pieces(i, o);
    const bool there = row < rows, live = 8 * i < r.dim && there, turning = 8 * i < o.rot;
    const int64_t at = row0 + row;

    auto fetch = [&](const T *x, v4 &a, v4 &b) {
        a = *reinterpret_cast<const v4 *>(x + p.a);
        b = *reinterpret_cast<const v4 *>(x + p.b);
    };
    const T *qx = (const T *)r.q + at * r.q_stride + (int64_t)h0 * r.dim, *kx = (const T *)r.k + at * r.k_stride + (int64_t)k0 * r.dim;
    v4 qa = {}, qb = {}, ka = {}, kb = {};     // lanes past the head keep zeros
    if (live && h0 < n_q) fetch(qx, qa, qb);
    if (live && k0 < n_k) fetch(kx, ka, kb);
    if (o.norm)
        for (int e = tid; e < r.dim; e += kThreads) {
            affine[e] = o.q_gain ? o.q_gain[e] : 1.f;
            affine[r.dim + e] = o.k_gain ? o.k_gain[e] : 1.f;
            affine[2 * r.dim + e] = o.q_shift ? o.q_shift[e] : 0.f;
            affine[3 * r.dim + e] = o.k_shift ? o.k_shift[e] : 0.f;
        }
    for (int t = tid; t < rows * pairs; t += kThreads) {
        const int tr = t / pairs, pi = t - tr * pairs;
        int axis = 0;
        while (axis + 1 < o.n_axes && pi >= o.axis_end[axis]) ++axis;
        cs[tr * pairs + (pi & 3) * quads + pi / 4] = unit(r.pos[(int64_t)(row0 + tr) * o.n_axes + axis], o.freq[pi]);
    }
    __syncthreads();
    const double2 *turns = cs + row * pairs + i;
    auto walk = [&](int h, int heads, const T *x, T *out, const float *gain, bool shifted, v4 a, v4 b) {
        const int64_t hop = (int64_t)step * r.dim;
        for (; h < heads; h += step) {
            asm volatile("" ::: "memory");       // factors are read from LDS for each head: kept in registers they would halve the waves
            double y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = (double)to_f32<T>(a[e]);
                y[4 + e] = (double)to_f32<T>(b[e]);
            }
            x += hop;
            if (live && h + step < heads) fetch(x, a, b);
            if (o.norm) {
                if (o.norm == 2) {
                    double s = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s += y[e];
                    const double mean = lanes_sum<L>(s) * sh.per_dim;
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = live ? y[e] - mean : 0.0;
                }
                double s = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fma(y[e], y[e], s);
                const double n_inv = rsqrt(fma(lanes_sum<L>(s), sh.per_dim, (double)o.eps));
                if (live) {
                    const f32x4 ga = *reinterpret_cast<const f32x4 *>(gain + p.a), gb = *reinterpret_cast<const f32x4 *>(gain + p.b);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[e] *= n_inv * (double)ga[e];
                        y[4 + e] *= n_inv * (double)gb[e];
                    }
                    if (shifted) {
                        const f32x4 sa = *reinterpret_cast<const f32x4 *>(gain + 2 * r.dim + p.a), sb = *reinterpret_cast<const f32x4 *>(gain + 2 * r.dim + p.b);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            y[e] += (double)sa[e];
                            y[4 + e] += (double)sb[e];
                        }
                    }
                }
            }
            if (!live) continue;
            if (turning) {
                if (o.adjacent) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) turn(y[2 * e], y[2 * e + 1], turns[e * quads]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) turn(y[e], y[4 + e], turns[e * quads]);
                }
            }
            store<T, 4>(out + p.a, round4<T>(y));
            store<T, 4>(out + p.b, round4<T>(y + 4));
            out += hop;
        }
    };
    walk(h0, n_q, qx, (T *)r.q_out + at * r.q_out_stride + (int64_t)h0 * r.dim, affine, o.q_shift, qa, qb);
    if constexpr (!WRITE) {
        walk(k0, n_k, kx, (T *)r.k_out + at * r.k_out_stride + (int64_t)k0 * r.dim, affine + r.dim, o.k_shift, ka, kb);
    } else {
        walk(k0, n_k, kx, keys + ((int64_t)row * r.n_kv + k0) * r.dim, affine + r.dim, o.k_shift, ka, kb);
        constexpr int AHEAD = 4;                // values requested before the first is needed
        const T *vx = (const T *)r.v + at * r.v_stride + (int64_t)h0 * r.dim + 8 * i;
        v8 xv[AHEAD];
#pragma unroll
        for (int w = 0; w < AHEAD; ++w)
            if (there && h0 + w * step < n_k) xv[w] = *reinterpret_cast<const v8 *>(vx + w * step * r.dim);
        const int32_t slot = there ? r.slot[at] : -1;
        const int off = slot & (kKv4Page - 1);
        __syncthreads();
        if (!there) return;
        uint8_t *blk = block_of(c, slot, h0);
        const T *key = keys + ((int64_t)row * r.n_kv + h0) * r.dim + 8 * i;
        for (int h = h0; h < n_k; h += AHEAD * step)
#pragma unroll
            for (int w = 0; w < AHEAD; ++w) {
                if (h + w * step >= n_k) break;
                hold_value<T>(blk, r.dim, off, i, xv[w]);
                if (h + (w + AHEAD) * step < n_k) xv[w] = *reinterpret_cast<const v8 *>(vx + (int64_t)(h - h0 + (w + AHEAD) * step) * r.dim);
                hold_key<T>(blk, r.dim, off, i, *reinterpret_cast<const v8 *>(key));
                if (blk) blk += (size_t)step * kv4_block_bytes(r.dim);
                key += step * r.dim;
            }
    }
}

// Keys and values as they are: eight channels of a token's key and value a thread, one head of rows that follow one another a workgroup, so that what it
// writes is the head's block of a page where the rows are its tokens.  40000 tokens of 16 heads of 64, 207 MB: 50 us in a row of calls on changing inputs, 4.2
// TB/s, and 61 in the kernel above (82 and 96 for scattered slots); right after a gigabyte of other writes 75, and 89 with all heads of a row side by
// side.  Requests for two or four rows at once (75 there) and value bytes exchanged between lanes for whole dwords (73) gave next to nothing.
template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_write_kernel(QkRows r, Kv4Cache c) {
    typedef typename Vec<T, 8>::v v8;
    const int chunks = r.dim / 8, h = blockIdx.y, ch = threadIdx.x % chunks;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / chunks) + threadIdx.x / chunks;
    if (row >= r.n_rows) return;
    const v8 k = *reinterpret_cast<const v8 *>((const T *)r.k + row * r.k_stride + (int64_t)h * r.dim + 8 * ch);
    const v8 v = *reinterpret_cast<const v8 *>((const T *)r.v + row * r.v_stride + (int64_t)h * r.dim + 8 * ch);
    const int32_t slot = r.slot[row];
    uint8_t *b = block_of(c, slot, h);
    hold_key<T>(b, r.dim, slot & (kKv4Page - 1), ch, k);
    hold_value<T>(b, r.dim, slot & (kKv4Page - 1), ch, v);
}

// Eight channels a thread, of a token's key and of its value; zeros for a slot outside the cache.  A workgroup takes one head of rows that follow
// one another: where these are a page's tokens it reads the head's block of the page whole, which workgroups on other XCDs would otherwise read
// again into their L2 (40000 tokens of 16 heads of 64: 53 us, 60 with two rows of all heads a workgroup).  Bound by memory: 54 us for those 207 MB, 3.9
// TB/s, four fifths of them writes; 4.4 us for 1000 scattered tokens.
constexpr int kReadAhead = 2;
template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(Kv4Cache c, const int32_t *slots, T *k, int64_t k_stride, T *v, int64_t v_stride,
                                                            int n_rows) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef T t2 __attribute__((ext_vector_type(2)));
    const int chunks = c.dim / 8, ng = c.dim / 32, h = blockIdx.y, ch = threadIdx.x % chunks, rows = kThreads / chunks;
    const int64_t row0 = (int64_t)blockIdx.x * rows * kReadAhead + threadIdx.x / chunks;
    uint32_t w[kReadAhead][2], sb[kReadAhead][2];
#pragma unroll
    for (int u = 0; u < kReadAhead; ++u) {
        const int64_t row = row0 + u * rows;
        const int32_t slot = row < n_rows ? slots[row] : -1;
        const uint8_t *b = block_of(c, slot, h);
        const int off = slot & (kKv4Page - 1);
        w[u][0] = w[u][1] = sb[u][0] = sb[u][1] = 0;
        if (b) {
            w[u][0] = *reinterpret_cast<const uint32_t *>(b + kv4_k_code(c.dim, off, ch));
            sb[u][0] = b[kv4_k_scale(c.dim, off, ch / 4)];
            const uint8_t *vb = b + kv4_v_code(c.dim, off, 4 * (ch % 4)) + ch / 4;
#pragma unroll
            for (int q = 0; q < 4; ++q) w[u][1] |= (uint32_t)vb[q * 4 * ng] << (8 * q);
            sb[u][1] = b[kv4_v_scale(c.dim, off) + ch / 4];
        }
    }
#pragma unroll
    for (int u = 0; u < kReadAhead; ++u) {
        const int64_t row = row0 + u * rows;
        if (row >= n_rows) return;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const float s = scale_of(sb[u][z]);
            const t2 x0 = __builtin_convertvector((f32x2)__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][z], s, 0), t2);
            const t2 x1 = __builtin_convertvector((f32x2)__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][z], s, 1), t2);
            const t2 x2 = __builtin_convertvector((f32x2)__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][z], s, 2), t2);
            const t2 x3 = __builtin_convertvector((f32x2)__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][z], s, 3), t2);
            T *out = (z ? v + row * v_stride : k + row * k_stride) + (int64_t)h * c.dim + 8 * ch;
            store<T, 8>(out, typename Vec<T, 8>::v{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]});
        }
    }
}

template <typename T, int L, bool WRITE>
void launch_rope_lanes(const QkOpts &o, const QkRows &r, const Kv4Cache &c, hipStream_t s) {
    constexpr int GROUPS = kThreads / L;
    const int heads = (r.q ? r.n_heads : 0) + (r.k ? r.n_kv : 0);
    // Rows of a workgroup: eight heads for a group, but 1024 workgroups where there are rows enough, and LDS that lets five share a CU
    const size_t row_lds = (size_t)(o.rot / 2) * sizeof(double2) + (WRITE ? (size_t)r.n_kv * r.dim * sizeof(T) : 0);
    int per = GROUPS;
    while (per > 1 && (per * heads > 8 * GROUPS || per > r.n_rows / 1024 || per * row_lds > 28672)) per /= 2;
    int log_step = 0;
    while (per << log_step < GROUPS) ++log_step;
    const RopeShape sh{per, log_step, 1.0 / r.dim};
    const dim3 grid((r.n_rows + per - 1) / per), block(kThreads);
    const size_t lds = per * row_lds + 4 * r.dim * sizeof(float);
    hipLaunchKernelGGL((qk_rope_kernel<T, L, WRITE>), grid, block, lds, s, o, r, c, sh);
}

template <typename T, bool WRITE>
void launch_rope(const QkOpts &o, const QkRows &r, const Kv4Cache &c, hipStream_t s) {
    if (r.dim <= 32) launch_rope_lanes<T, 4, WRITE>(o, r, c, s);
    else if (r.dim <= 64) launch_rope_lanes<T, 8, WRITE>(o, r, c, s);
    else if (r.dim <= 128) launch_rope_lanes<T, 16, WRITE>(o, r, c, s);
    else launch_rope_lanes<T, 32, WRITE>(o, r, c, s);
}

}  // namespace

template <typename T> void launch_qk_rope(const QkOpts &o, const QkRows &r, hipStream_t s) {
    if (r.n_rows > 0) launch_rope<T, false>(o, r, Kv4Cache{}, s);
}

template <typename T> void launch_kv4_write(const Kv4Cache &c, const QkOpts *o, const QkRows &r, hipStream_t s) {
    if (r.n_rows <= 0) return;
    if (o) return launch_rope<T, true>(*o, r, c, s);
    const int rows = kThreads / (r.dim / 8);
    hipLaunchKernelGGL((kv4_write_kernel<T>), dim3((r.n_rows + rows - 1) / rows, r.n_kv), dim3(kThreads), 0, s, r, c);
}

template <typename T> void launch_kv4_read(const Kv4Cache &c, const int32_t *slot, void *k, int64_t k_stride, void *v, int64_t v_stride,
                                           int n_rows, hipStream_t s) {
    if (n_rows <= 0) return;
    const int rows = kThreads / (c.dim / 8) * kReadAhead;
    const dim3 grid((n_rows + rows - 1) / rows, c.n_heads), block(kThreads);
    hipLaunchKernelGGL((kv4_read_kernel<T>), grid, block, 0, s, c, slot, (T *)k, k_stride, (T *)v, v_stride, n_rows);
}

#define SJD_KV4_ROWS(T)                                                                                     \
    template void launch_qk_rope<T>(const QkOpts &, const QkRows &, hipStream_t);                           \
    template void launch_kv4_write<T>(const Kv4Cache &, const QkOpts *, const QkRows &, hipStream_t);       \
    template void launch_kv4_read<T>(const Kv4Cache &, const int32_t *, void *, int64_t, void *, int64_t, int, hipStream_t);
SJD_KV4_ROWS(float)
SJD_KV4_ROWS(bf16)
SJD_KV4_ROWS(f16)

}  // namespace sjd
