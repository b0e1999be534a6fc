// Rows normed and held in 8 bits, with the residual's addition in front, and 8-bit rows read back.
//
//   h = round(resid + x)  ->  resid            (where there is a residual; else h = x)
//   y = h / sqrt(mean h^2 + eps) * gain + shift      or      (h - mean) / sqrt(mean (h - mean)^2 + eps) * gain + shift      or      h
//   out = 8 bits of float32(y), a power of two for each 128 channels (f8.h)
//
// Everything between h and the rounding to float32 is float64: a value next to a border of the 8-bit grid then goes to its side in whatever order sums
// are taken.  The vector unit does float64 at the rate of float32, and the kernel moves bytes: each row is read once, held in registers, written once.
#include "f8.h"
#include "gemm_rules.h"

namespace sjd {

namespace {

template <typename T> struct Vec8 { typedef T v __attribute__((ext_vector_type(8), aligned(sizeof(T)))); };

// Eight values from p on, those from `left` on as zeros.
template <typename T> __device__ __forceinline__ void load8(const T *p, int left, float (&h)[8]) {
    if (left >= 8) {
        const typename Vec8<T>::v v = *reinterpret_cast<const typename Vec8<T>::v *>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = to_f32(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = e < left ? to_f32(p[e]) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, int left, const float (&h)[8]) {
    if (left >= 8) {
        typename Vec8<T>::v v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = from_f32<T>(h[e]);
        *reinterpret_cast<typename Vec8<T>::v *>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = from_f32<T>(h[e]);
    }
}

template <int CTRL> __device__ __forceinline__ double dpp_add(double v) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 x = __builtin_bit_cast(i32x2, v);
    const i32x2 y = {__builtin_amdgcn_update_dpp(0, x.x, CTRL, 0xf, 0xf, true), __builtin_amdgcn_update_dpp(0, x.y, CTRL, 0xf, 0xf, true)};
    return v + __builtin_bit_cast(double, y);
}
// The sum over the L lanes (16, 32, 64) and W waves of a row, the same in all of them: quads by permutation, then mirrors, then rows of sixteen and halves swapped.
template <int L, int W> __device__ __forceinline__ double row_sum(double v, double *parts) {
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    v = dpp_add<0x140>(v);
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    auto fold = [](double d, auto swap) {
        const u32x2 x = __builtin_bit_cast(u32x2, d);
        const auto lo = swap(x.x), hi = swap(x.y);
        return __builtin_bit_cast(double, (u32x2{lo[0], hi[0]})) + __builtin_bit_cast(double, (u32x2{lo[1], hi[1]}));
    };
    if constexpr (L >= 32) v = fold(v, [](unsigned q) { return __builtin_amdgcn_permlane16_swap(q, q, false, false); });
    if constexpr (L >= 64) v = fold(v, [](unsigned q) { return __builtin_amdgcn_permlane32_swap(q, q, false, false); });
    if constexpr (W > 1) {
        __syncthreads();                                   // the parts of an earlier sum have been read
        if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) v += parts[w];
    }
    return v;
}

// L lanes and W waves a row (W = 1: 256 / L rows a workgroup), CH pieces of eight channels a lane.  NORM: 0 none, 1 root mean square, 2 mean and variance.  Gains and
// shifts are requested with the row: after the sums they would be another trip to memory.
// Bound by memory where rows are many: 32768 x 1024 in half with a float32 stream 75 us, 4.9 TB/s of the 5.1 that a copy of 1 GiB reaches; 20000 x 1024 of float32 without a norm
// 20 us, 5.0.  4999 x 2001 with mean and variance 24 us: two sums in turn, each over the four waves of a row.  32 rows of 1024 4.6 us, a launch and one trip.
template <typename T, typename R, bool RESID, int NORM, int L, int W, int CH>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void norm_f8_kernel(NormF8 a) {
    __shared__ double parts[W];
    constexpr int LANES = W == 1 ? L : 64 * W;
    const int tid = threadIdx.x % LANES;
    const int64_t row = W == 1 ? (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L : blockIdx.x;
    if (row >= a.out.n_rows) return;                       // whole rows leave
    const int width = a.out.width;
    const T *x = (const T *)a.x + row * a.x_stride;
    R *r = RESID ? (R *)a.resid + row * a.resid_stride : nullptr;
    constexpr bool EARLY = CH <= 2;                        // as far as registers go
    float h[CH][8], gain[NORM && EARLY ? CH : 1][8], shift[NORM == 2 && EARLY ? CH : 1][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (c * LANES + tid) * 8;
        load8(x + at, width - at, h[c]);
        if constexpr (NORM && EARLY) {
            if (a.gain) load8(a.gain + at, width - at, gain[c]);
        }
        if constexpr (NORM == 2 && EARLY) {
            if (a.shift) load8(a.shift + at, width - at, shift[c]);
        }
        if constexpr (RESID) {
            float q[8];
            load8(r + at, width - at, q);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[c][e] = to_f32(from_f32<R>(keep_f32(q[e] + h[c][e])));
        }
    }
    if constexpr (RESID) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (c * LANES + tid) * 8;
            store8(r + at, width - at, h[c]);
        }
    }
    double mean = 0, inv = 1;
    if constexpr (NORM == 2) {
        double s = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += (double)h[c][e];
        mean = row_sum<L, W>(s, parts) / width;
    }
    if constexpr (NORM) {
        double s = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (c * LANES + tid) * 8;
            if (NORM == 1 || at + 8 <= width) {            // zeros behind the row add nothing to a sum of squares
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double d = NORM == 2 ? (double)h[c][e] - mean : (double)h[c][e];
                    s = fma(d, d, s);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double d = at + e < width ? (double)h[c][e] - mean : 0.0;
                    s = fma(d, d, s);
                }
            }
        }
        inv = 1.0 / sqrt(row_sum<L, W>(s, parts) / width + a.eps);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (c * LANES + tid) * 8;
        if constexpr (NORM) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                double y = NORM == 2 ? ((double)h[c][e] - mean) * inv : (double)h[c][e] * inv;
                if constexpr (EARLY) {
                    if (a.gain) y *= (double)gain[c][e];
                } else if (a.gain && at + e < width) {
                    y *= (double)a.gain[at + e];
                }
                if constexpr (NORM == 2 && EARLY) {
                    if (a.shift) y += (double)shift[c][e];
                } else if (a.shift && at + e < width) {
                    y += (double)a.shift[at + e];
                }
                h[c][e] = (float)y;
            }
            if (at + 8 > width) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[c][e] = at + e < width ? h[c][e] : 0.f;
            }
        }
        f8_hold8(a.out, row, at, h[c]);
    }
}

template <typename T, typename R, bool RESID, int NORM> void launch_norm_of(const NormF8 &a, hipStream_t s) {
    const int n = a.out.n_rows, w = a.out.width;
    if (w <= 128) norm_f8_kernel<T, R, RESID, NORM, 16, 1, 1><<<(n + 15) / 16, 256, 0, s>>>(a);
    else if (w <= 256) norm_f8_kernel<T, R, RESID, NORM, 32, 1, 1><<<(n + 7) / 8, 256, 0, s>>>(a);
    else if (w <= 512) norm_f8_kernel<T, R, RESID, NORM, 64, 1, 1><<<(n + 3) / 4, 256, 0, s>>>(a);
    else if (w <= 1024) norm_f8_kernel<T, R, RESID, NORM, 64, 1, 2><<<(n + 3) / 4, 256, 0, s>>>(a);
    else if (w <= 2048) norm_f8_kernel<T, R, RESID, NORM, 64, 4, 1><<<n, 256, 0, s>>>(a);
    else if (w <= 4096) norm_f8_kernel<T, R, RESID, NORM, 64, 8, 1><<<n, 512, 0, s>>>(a);
    else if (w <= 8192) norm_f8_kernel<T, R, RESID, NORM, 64, 8, 2><<<n, 512, 0, s>>>(a);
    else if (w <= 16384) norm_f8_kernel<T, R, RESID, NORM, 64, 16, 2><<<n, 1024, 0, s>>>(a);
    else norm_f8_kernel<T, R, RESID, NORM, 64, 16, 4><<<n, 1024, 0, s>>>(a);
}
template <typename T, typename R, bool RESID> void launch_norm_by(const NormF8 &a, hipStream_t s) {
    if (a.norm == 0) launch_norm_of<T, R, RESID, 0>(a, s);
    else if (a.norm == 1) launch_norm_of<T, R, RESID, 1>(a, s);
    else launch_norm_of<T, R, RESID, 2>(a, s);
}

// Eight values a lane, `lanes` of them (a power of two) a row.  Bound by memory: 32768 x 1024 to half 17 us, 5.8 TB/s (part of it from the last-level cache).
template <typename T> __global__ __launch_bounds__(256) void f8_read_kernel(F8Rows r, T *out, int64_t stride, int lanes) {
    const int per = 256 / lanes;
    const int64_t row = (int64_t)blockIdx.x * per + threadIdx.x / lanes;
    if (row >= r.n_rows) return;
    for (int at = (threadIdx.x % lanes) * 8; at < r.width; at += lanes * 8) {
        const uint2 c = *reinterpret_cast<const uint2 *>(r.codes + row * r.code_stride + at);
        const float s = f8_scale(r.scales[row * r.scale_stride + at / kF8Group]);
        float h[8];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t w = q ? c.y : c.x;
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, true);
            h[4 * q] = lo[0]; h[4 * q + 1] = lo[1]; h[4 * q + 2] = hi[0]; h[4 * q + 3] = hi[1];
        }
        store8(out + row * stride + at, r.width - at, h);
    }
}

}  // namespace

template <typename T> void launch_norm_f8(const NormF8 &a, bool resid_f32, hipStream_t s) {
    if (!a.resid) launch_norm_by<T, float, false>(a, s);
    else if (resid_f32) launch_norm_by<T, float, true>(a, s);
    else launch_norm_by<T, T, true>(a, s);
}
template void launch_norm_f8<float>(const NormF8 &, bool, hipStream_t);
template void launch_norm_f8<bf16>(const NormF8 &, bool, hipStream_t);
template void launch_norm_f8<f16>(const NormF8 &, bool, hipStream_t);

template <typename T> void launch_f8_read(const F8Rows &r, T *out, int64_t stride, hipStream_t s) {
    const int lanes = f8_read_lanes(r.width, r.n_rows), per = 256 / lanes;
    f8_read_kernel<T><<<(int)(((int64_t)r.n_rows + per - 1) / per), 256, 0, s>>>(r, out, stride, lanes);
}
template void launch_f8_read<float>(const F8Rows &, float *, int64_t, hipStream_t);
template void launch_f8_read<bf16>(const F8Rows &, bf16 *, int64_t, hipStream_t);
template void launch_f8_read<f16>(const F8Rows &, f16 *, int64_t, hipStream_t);

}  // namespace sjd
