// Queries and keys normed for each head and rotated by their positions, and the cache of 4 bits written and read.
//
//   y = x / sqrt(mean x^2 + eps) * gain      or      (x - mean) / sqrt(var + eps) * gain + shift      (over the channels of a head)
//   (y_a, y_b) <- (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = position[axis of the pair] * frequency[pair]
//
// Everything between the load and the one rounding to the rows' type is float64: a value that lands next to a border of the 4-bit
// grid then goes to the same side in whatever order sums are taken (float32 sums in another order move one key in ten million to
// the next level, a third of its size), and angles of far positions keep their digits.  The vector unit does float64 at the rate
// of float32 here, and these kernels move bytes: each row is read once and written once.
#include "kv4.h"

namespace sjd {

namespace {

// cos and sin of p * f in float64.  The product of a 32-bit integer and a float32 needs 55 bits: taken as a sum of two doubles,
// and so are the turns p f / 2 pi, of which the whole ones go; the fraction is good to 2^-52 of a turn.
__device__ __forceinline__ double2 unit(int32_t p, float f) {
#pragma clang fp contract(off)   // th below is the rounded product, also where it is subtracted from
    const double ah = (double)p * (double)f, al = fma((double)p, (double)f, -ah);
    const double ih = 0.15915494309189535, il = -9.839338337591243e-18;     // 1 / 2 pi
    const double th = ah * ih, tl = fma(ah, ih, -th) + fma(ah, il, al * ih);
    double s, c;
    sincospi(2.0 * ((th - rint(th)) + tl), &s, &c);
    return {c, s};
}

// four values that start on a multiple of their own size
template <typename T> __device__ __forceinline__ void load4(const T *p, float (&x)[4]) {
    typedef T v4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const v4 t = *reinterpret_cast<const v4 *>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = to_f32<T>(t[e]);
}
template <typename T> __device__ __forceinline__ void store4(T *p, const T (&x)[4]) {
    typedef T v4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    *reinterpret_cast<v4 *>(p) = v4{x[0], x[1], x[2], x[3]};
}

template <int L> __device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Where a lane's two pieces of four channels begin: piece b holds the partners of piece a where the pairs are rot / 2 apart.
struct Pieces { int a, b; };
__device__ __forceinline__ Pieces pieces(int i, const QkOpts &o) {
    if (!o.adjacent && 8 * i < o.rot) return {4 * i, 4 * i + o.rot / 2};
    return {8 * i, 8 * i + 4};
}

__device__ __forceinline__ void turn(double &a, double &b, double2 u) {
    const double x = a;
    a = fma(x, u.x, -(b * u.y));
    b = fma(b, u.x, x * u.y);
}

// One head of one row on L lanes (lane i of them): norm and rotation of the lane's eight channels.
template <int L>
__device__ __forceinline__ void head_turn(const QkOpts &o, int dim, int i, Pieces p, const float (&xa)[4], const float (&xb)[4],
                                          const float *gain, const float *shift, const double2 *cs, double (&y)[8]) {
    const bool live = 8 * i < dim;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = live ? (double)xa[e] : 0.0;
        y[4 + e] = live ? (double)xb[e] : 0.0;
    }
    if (o.norm) {
        if (o.norm == 2) {
            double s = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += y[e];
            const double mean = lanes_sum<L>(s) / dim;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = live ? y[e] - mean : 0.0;
        }
        double s = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma(y[e], y[e], s);
        const double r = rsqrt(lanes_sum<L>(s) / dim + (double)o.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= r;
        if (gain && live) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] *= (double)gain[p.a + e];
                y[4 + e] *= (double)gain[p.b + e];
            }
        }
        if (shift && live) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] += (double)shift[p.a + e];
                y[4 + e] += (double)shift[p.b + e];
            }
        }
    }
    if (8 * i < o.rot) {
        if (o.adjacent) {
#pragma unroll
            for (int e = 0; e < 4; ++e) turn(y[2 * e], y[2 * e + 1], cs[4 * i + e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) turn(y[e], y[4 + e], cs[4 * i + e]);
        }
    }
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
__device__ __forceinline__ uint32_t encode2(float a, float b, uint32_t byte) {
    if (byte == 255) return 0;
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale_of(byte), 0) & 255u;
}
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <int L> __device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}

// Where a token's block is, nullptr where the slot is outside the cache.
__device__ __forceinline__ uint8_t *block_of(const Kv4Cache &c, int32_t slot, int head) {
    if (slot < 0 || slot >= (int64_t)c.n_pages * kKv4Page) return nullptr;
    return c.pages + ((size_t)(slot / kKv4Page) * c.n_heads + head) * kv4_block_bytes(c.dim);
}

// ---- kernels ---------------------------------------------------------------------------------

constexpr int kThreads = 256;

// A workgroup takes `per` rows.  First every (row, pair) gets its cos and sin, once for all heads; then L lanes a head, all heads of its
// rows.  WRITE: keys go to LDS, rounded to their type, instead of memory, and with the values from there into the cache.
template <typename T, int L, bool WRITE>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(QkOpts o, QkRows r, Kv4Cache c, int per) {
    extern __shared__ char smem[];
    double2 *cs = reinterpret_cast<double2 *>(smem);
    const int pairs = o.rot / 2;
    T *keys = reinterpret_cast<T *>(smem + (size_t)per * pairs * sizeof(double2));      // [per][n_kv][dim]
    const int row0 = blockIdx.x * per, rows = min(per, r.n_rows - row0);
    const int tid = threadIdx.x;
    for (int t = tid; t < rows * pairs; t += kThreads) {
        const int row = t / pairs, i = t - row * pairs;
        int axis = 0;
        while (axis + 1 < o.n_axes && i >= o.axis_end[axis]) ++axis;
        cs[t] = unit(r.pos[(int64_t)(row0 + row) * o.n_axes + axis], o.freq[i]);
    }
    __syncthreads();
    const int i = tid % L, heads = (r.q ? r.n_heads : 0) + (r.k ? r.n_kv : 0);
    const Pieces p = pieces(i, o);
    const bool live = 8 * i < r.dim;
    for (int t = tid / L; t < rows * heads; t += kThreads / L) {
        const int row = t / heads, hh = t - row * heads;
        const bool is_q = r.q && hh < r.n_heads;
        const int h = is_q ? hh : hh - (r.q ? r.n_heads : 0);
        const int64_t at = row0 + row;
        const T *x = is_q ? (const T *)r.q + at * r.q_stride + (int64_t)h * r.dim : (const T *)r.k + at * r.k_stride + (int64_t)h * r.dim;
        float xa[4] = {}, xb[4] = {};
        if (live) {
            load4<T>(x + p.a, xa);
            load4<T>(x + p.b, xb);
        }
        double y[8];
        head_turn<L>(o, r.dim, i, p, xa, xb, is_q ? o.q_gain : o.k_gain, is_q ? o.q_shift : o.k_shift, cs + row * pairs, y);
        if (!live) continue;
        T ya[4], yb[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ya[e] = from_f32<T>((float)y[e]);
            yb[e] = from_f32<T>((float)y[4 + e]);
        }
        if (WRITE && !is_q) {
            T *k = keys + ((size_t)row * r.n_kv + h) * r.dim;
            store4<T>(k + p.a, ya);
            store4<T>(k + p.b, yb);
        } else {
            T *out = is_q ? (T *)r.q_out + at * r.q_out_stride + (int64_t)h * r.dim : (T *)r.k_out + at * r.k_out_stride + (int64_t)h * r.dim;
            store4<T>(out + p.a, ya);
            store4<T>(out + p.b, yb);
        }
    }
    if constexpr (WRITE) {
        __syncthreads();
        const int ng = r.dim / 32, chunks = r.dim / 8;
        // keys: eight channels a lane, four lanes a group (their number is a multiple of four: a group's lanes stay together)
        for (int t = tid; t < rows * r.n_kv * chunks; t += kThreads) {
            const int row = t / (r.n_kv * chunks), rest = t - row * r.n_kv * chunks, h = rest / chunks, ch = rest - h * chunks;
            float x[8];
            const T *k = keys + ((size_t)row * r.n_kv + h) * r.dim + 8 * ch;
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = to_f32<T>(k[e]); top = max(top, mag(x[e])); }
            top = lanes_max<4>(top);
            const int32_t slot = r.slot[row0 + row];
            uint8_t *b = block_of(c, slot, h);
            if (!b) continue;
            const int off = slot % kKv4Page;
            const uint32_t sb = scale_byte<T>(top);
            *reinterpret_cast<uint32_t *>(b + kv4_k_code(r.dim, off, ch)) = encode8(x, sb);
            if (ch % 4 == 0) b[kv4_k_scale(r.dim, off, ch / 4)] = (uint8_t)sb;
        }
        // values: sixteen lanes a token and head, a channel pair of each group
        for (int t = tid; t < rows * r.n_kv * 16; t += kThreads) {
            const int row = t / (r.n_kv * 16), rest = t - row * r.n_kv * 16, h = rest / 16, n = rest % 16;
            const int32_t slot = r.slot[row0 + row];
            uint8_t *b = block_of(c, slot, h);
            const int off = slot % kKv4Page;
            const T *v = (const T *)r.v + (int64_t)(row0 + row) * r.v_stride + (int64_t)h * r.dim + 2 * n;
            for (int g = 0; g < ng; ++g) {
                const float x0 = to_f32<T>(v[32 * g]), x1 = to_f32<T>(v[32 * g + 1]);
                const uint32_t sb = scale_byte<T>(lanes_max<16>(max(mag(x0), mag(x1))));
                if (!b) continue;
                b[kv4_v_code(r.dim, off, n) + g] = (uint8_t)encode2(x0, x1, sb);
                if (n == 0) b[kv4_v_scale(r.dim, off) + g] = (uint8_t)sb;
            }
        }
    }
}

// keys and values as they are
template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_write_kernel(QkRows r, Kv4Cache c) {
    const int ng = r.dim / 32, chunks = r.dim / 8;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t n_k = (int64_t)r.n_rows * r.n_kv * chunks;
    const int64_t k_blocks = (n_k + kThreads - 1) / kThreads * kThreads;
    if (id < k_blocks) {
        if (id >= n_k) return;
        const int64_t row = id / (r.n_kv * chunks);
        const int rest = (int)(id - row * r.n_kv * chunks), h = rest / chunks, ch = rest - h * chunks;
        const T *k = (const T *)r.k + row * r.k_stride + (int64_t)h * r.dim + 8 * ch;
        float x[8];
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[e] = to_f32<T>(k[e]); top = max(top, mag(x[e])); }
        top = lanes_max<4>(top);
        const int32_t slot = r.slot[row];
        uint8_t *b = block_of(c, slot, h);
        if (!b) return;
        const int off = slot % kKv4Page;
        const uint32_t sb = scale_byte<T>(top);
        *reinterpret_cast<uint32_t *>(b + kv4_k_code(r.dim, off, ch)) = encode8(x, sb);
        if (ch % 4 == 0) b[kv4_k_scale(r.dim, off, ch / 4)] = (uint8_t)sb;
        return;
    }
    const int64_t t = id - k_blocks;
    if (t >= (int64_t)r.n_rows * r.n_kv * 16) return;
    const int64_t row = t / (r.n_kv * 16);
    const int rest = (int)(t - row * r.n_kv * 16), h = rest / 16, n = rest % 16;
    const int32_t slot = r.slot[row];
    uint8_t *b = block_of(c, slot, h);
    const int off = slot % kKv4Page;
    const T *v = (const T *)r.v + row * r.v_stride + (int64_t)h * r.dim + 2 * n;
    for (int g = 0; g < ng; ++g) {
        const float x0 = to_f32<T>(v[32 * g]), x1 = to_f32<T>(v[32 * g + 1]);
        const uint32_t sb = scale_byte<T>(lanes_max<16>(max(mag(x0), mag(x1))));
        if (!b) continue;
        b[kv4_v_code(r.dim, off, n) + g] = (uint8_t)encode2(x0, x1, sb);
        if (n == 0) b[kv4_v_scale(r.dim, off) + g] = (uint8_t)sb;
    }
}

// eight channels a lane: of the keys of a token, then of its values; zeros for a slot outside the cache
template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(Kv4Cache c, const int32_t *slots, T *k, int64_t k_stride, T *v, int64_t v_stride,
                                                            int n_rows) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const int chunks = c.dim / 8;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = id / (c.n_heads * chunks);
    if (row >= n_rows) return;
    const int rest = (int)(id - row * c.n_heads * chunks), h = rest / chunks, ch = rest - h * chunks;
    const int32_t slot = slots[row];
    const uint8_t *b = block_of(c, slot, h);
    const int off = slot % kKv4Page;
    uint32_t w[2] = {0, 0}, sb[2] = {0, 0};
    if (b) {
        w[0] = *reinterpret_cast<const uint32_t *>(b + kv4_k_code(c.dim, off, ch));
        sb[0] = b[kv4_k_scale(c.dim, off, ch / 4)];
        for (int q = 0; q < 4; ++q) w[1] |= (uint32_t)b[kv4_v_code(c.dim, off, 4 * (ch % 4) + q) + ch / 4] << (8 * q);
        sb[1] = b[kv4_v_scale(c.dim, off) + ch / 4];
    }
    T *out[2] = {k + row * k_stride + (int64_t)h * c.dim + 8 * ch, v + row * v_stride + (int64_t)h * c.dim + 8 * ch};
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const float s = scale_of(sb[z]);
        f32x2 x[4];
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[z], s, 0);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[z], s, 1);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[z], s, 2);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[z], s, 3);
#pragma unroll
        for (int e = 0; e < 8; ++e) out[z][e] = from_f32<T>(x[e / 2][e % 2]);
    }
}

template <typename T, bool WRITE>
void launch_rope(const QkOpts &o, const QkRows &r, const Kv4Cache &c, hipStream_t s) {
    const size_t row_lds = (size_t)(o.rot / 2) * sizeof(double2) + (WRITE ? (size_t)r.n_kv * r.dim * sizeof(T) : 0);
    const int per = r.n_rows >= 4096 && 4 * row_lds <= 32768 ? 4 : 1;
    const size_t lds = per * row_lds;
    const dim3 grid((r.n_rows + per - 1) / per);
    if (r.dim <= 32) hipLaunchKernelGGL((qk_rope_kernel<T, 4, WRITE>), grid, dim3(kThreads), lds, s, o, r, c, per);
    else if (r.dim <= 64) hipLaunchKernelGGL((qk_rope_kernel<T, 8, WRITE>), grid, dim3(kThreads), lds, s, o, r, c, per);
    else if (r.dim <= 128) hipLaunchKernelGGL((qk_rope_kernel<T, 16, WRITE>), grid, dim3(kThreads), lds, s, o, r, c, per);
    else hipLaunchKernelGGL((qk_rope_kernel<T, 32, WRITE>), grid, dim3(kThreads), lds, s, o, r, c, per);
}

}  // namespace

template <typename T> void launch_qk_rope(const QkOpts &o, const QkRows &r, hipStream_t s) {
    if (r.n_rows > 0) launch_rope<T, false>(o, r, Kv4Cache{}, s);
}

template <typename T> void launch_kv4_write(const Kv4Cache &c, const QkOpts *o, const QkRows &r, hipStream_t s) {
    if (r.n_rows <= 0) return;
    if (o) return launch_rope<T, true>(*o, r, c, s);
    const int64_t nk = ((int64_t)r.n_rows * r.n_kv * (r.dim / 8) + kThreads - 1) / kThreads;
    const int64_t nv = ((int64_t)r.n_rows * r.n_kv * 16 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((kv4_write_kernel<T>), dim3((unsigned)(nk + nv)), dim3(kThreads), 0, s, r, c);
}

template <typename T> void launch_kv4_read(const Kv4Cache &c, const int32_t *slot, void *k, int64_t k_stride, void *v, int64_t v_stride,
                                           int n_rows, hipStream_t s) {
    if (n_rows <= 0) return;
    const int64_t n = ((int64_t)n_rows * c.n_heads * (c.dim / 8) + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((kv4_read_kernel<T>), dim3((unsigned)n), dim3(kThreads), 0, s, c, slot, (T *)k, k_stride, (T *)v, v_stride, n_rows);
}

#define SJD_KV4_ROWS(T)                                                                                     \
    template void launch_qk_rope<T>(const QkOpts &, const QkRows &, hipStream_t);                           \
    template void launch_kv4_write<T>(const Kv4Cache &, const QkOpts *, const QkRows &, hipStream_t);       \
    template void launch_kv4_read<T>(const Kv4Cache &, const int32_t *, void *, int64_t, void *, int64_t, int, hipStream_t);
SJD_KV4_ROWS(float)
SJD_KV4_ROWS(bf16)
SJD_KV4_ROWS(f16)

}  // namespace sjd
