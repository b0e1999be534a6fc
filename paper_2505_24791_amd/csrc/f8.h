// Rows held in 8 bits: format, conversions, launchers (norm_f8.hip, gemm_f8.hip).
//
// A row of `width` values is held as 8-bit floats (4 exponent bits, bias 7, 3 mantissa bits; largest 448, 0x7f and 0xff not a number), padded with
// zeros to a multiple of 128.  128 consecutive values share a power of two s = 2^e, held as the byte e + 127: the smallest s with
// max |x| <= 448 s over the finite values, -120 <= e <= 120.  A power of two takes no bits from the values, the matrix unit
// multiplies by it for nothing, and conversions to and from it are single instructions; a float32 scale would have to be multiplied
// into every 128 products' sum by the vector unit.  The four scales of 512 values are one dword of a row.
#pragma once
#include "common.h"

namespace sjd {

constexpr int kF8Group = 128;

struct F8Rows {
    uint8_t *codes, *scales;
    int64_t code_stride, scale_stride;      // bytes
    int n_rows, width;
    __host__ __device__ int groups() const { return (width + kF8Group - 1) / kF8Group; }
};

// Norm and hold: h = x (+ resid, rounded to the residual's type and stored there), out = 8 bits of norm(h) * gain + shift.
struct NormF8 {
    const void *x;
    void *resid;                    // nullable
    int64_t x_stride, resid_stride; // elements
    const float *gain, *shift;      // [width], nullptr: 1, 0
    double eps;
    int norm;                       // 0 none, 1 x / sqrt(mean x^2 + eps), 2 (x - mean) / sqrt(var + eps)
    F8Rows out;
};
constexpr int kNormF8Most = 32768;  // widest row
// T: rows; resid_f32: the residual is float32, else of type T
template <typename T> void launch_norm_f8(const NormF8 &a, bool resid_f32, hipStream_t s);
// values back in T
template <typename T> void launch_f8_read(const F8Rows &r, T *out, int64_t stride, hipStream_t s);

// The exponent byte of a group from the bits of its largest finite magnitude.  448 = 1.75 * 2^8: a mantissa above 1.75 takes the next power.
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t top) {
    const int e = (int)((top + 0x1fffffu) >> 23) - 8;
    return (uint32_t)min(max(e, 127 - 120), 127 + 120);
}
__device__ __forceinline__ float f8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight values in 8 bits each, times 2^-(byte - 127), to nearest even.  Infinities and NaN become NaN.
__device__ __forceinline__ uint2 f8_encode8(const float (&x)[8], uint32_t byte) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const float s = f8_scale(byte);
    s16x2 a = {0, 0}, b = {0, 0};
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[0], x[1], s, false);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[2], x[3], s, true);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[4], x[5], s, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[6], x[7], s, true);
    return {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}

// the bits of |x|, 0 where it is not finite
__device__ __forceinline__ uint32_t f8_finite_mag(float x) {
    const uint32_t m = __float_as_uint(x) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
}

// the largest over 16 neighbouring lanes: quads by permutation, then mirrors
__device__ __forceinline__ uint32_t f8_max16(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));
}

// Eight consecutive values (a sixteenth of a group; the sixteen lanes of a group are neighbours) into a row: `at` is their first channel.
// Channels after the end of the row come as zeros.
__device__ __forceinline__ void f8_hold8(const F8Rows &r, int64_t row, int at, const float (&x)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, f8_finite_mag(x[e]));
    top = f8_max16(top);
    const uint32_t byte = f8_scale_byte(top);
    const int groups = r.groups(), group = at / kF8Group;
    if (group < groups) *reinterpret_cast<uint2 *>(r.codes + row * r.code_stride + at) = f8_encode8(x, byte);
    if (at % kF8Group == 0 && group < groups) {
        uint8_t *s = r.scales + row * r.scale_stride + group;
        *s = (uint8_t)byte;
        if (group == groups - 1)
            for (int q = 1; (group + q) & 3; ++q) s[q] = 0;
    }
}

// C = rows * weight^T + bias, in T (16 bits) or float32; accumulate (float32): C += .
struct LinearF8 {
    F8Rows x, w;
    const float *bias;              // nullable
    void *c;
    int64_t c_stride;               // elements
    int dtype;                      // of C, SJD_DTYPE_*
    bool accumulate;
};
void launch_linear_f8(const LinearF8 &a, hipStream_t s);

// hidden = 8 bits of act(x gate^T) * (x up^T); w: the rows of gate, then those of up
struct GatedF8 {
    F8Rows x, w, hidden;
    float *loose;                   // [rows][loose_stride] where gated_f8_holds() is false: the hidden rows in float32, on their way
    int64_t loose_stride;           // the hidden channels rounded up to four
    int act;                        // 0 x * sigmoid(x), 1 GELU (erf)
    int dtype;                      // of the results behind them, SJD_DTYPE_*: which sums the hidden rows are of (see gemm_f8.hip)
};
void launch_gated_f8(const GatedF8 &a, hipStream_t s);
// Whether the product's own launch holds the hidden rows in 8 bits: it has whole groups of 128 channels in a workgroup, as the launch for few rows and short k and those for 16-bit
// results that fill the chip do.
bool gated_f8_holds(const F8Rows &x, const F8Rows &w, int dtype);

}  // namespace sjd
