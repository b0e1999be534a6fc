// Projections of 8-bit rows by 8-bit weights, C = X W^T + bias, and the first half of the gated block, hidden = act(X G^T) * (X U^T) in 8 bits.
//
// 16-bit results: the 32x32x64 instruction on the codes, which multiplies each operand's row by its scale as it goes.  Of eight products at a time it
// drops what lies 2^-14 or more below the largest; sums of those eights are float32.  Against 64 bits that is 1.4e-5 (relative, 2-norm, normal
// operands), 1e-2 of what bfloat16 results are rounded by and 7e-2 for half.
// float32 results (EXACT): code times scale is a bfloat16 number, converted in registers, and the 32x32x16 bfloat16 instruction sums exact
// products in float32, at half the rate.
#include "f8.h"
#include "gemm_rules.h"
#include <atomic>
#include <type_traits>

namespace sjd {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

#define SJD_F8_LPTR(p) ((__attribute__((address_space(3))) void *)(p))

template <int N> __device__ __forceinline__ void wait_loads() {          // vmcnt(N) lgkmcnt(0)
    __builtin_amdgcn_s_waitcnt((N & 15) | 0x70 | ((N >> 4) << 14));
}

// 64 lanes x 16 (4) bytes from a wave-uniform base plus a 32-bit lane offset to 1 KB (256 bytes) of LDS at the wave-uniform address.  M0 is set inside the
// statement and nothing else in these kernels reads it.  Five wait states before the load: the compiler does not look into the statement, and where it keeps the
// base in lanes of a vector register, the scalar registers it has just been read back into are not there for a memory instruction any sooner.
__device__ __forceinline__ void dma16(const void *base, uint32_t off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void dma4(const void *base, uint32_t off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_addr), "v"(off), "s"(base) : "memory");
}

__device__ __forceinline__ i32x8 join(i32x4 a, i32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// sixteen codes times their scale, eight values a half in the order of the codes
struct Half2 { bf16x8 v[2]; };
__device__ __forceinline__ Half2 widen(i32x4 c, float s) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    Half2 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const b2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[q], s, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[q], s, true);
        const int o = 4 * (q & 1);
        r.v[q >> 1][o] = lo[0]; r.v[q >> 1][o + 1] = lo[1]; r.v[q >> 1][o + 2] = hi[0]; r.v[q >> 1][o + 3] = hi[1];
    }
    return r;
}

// Lets a kernel have `bytes` of dynamic LDS, once for each device (bit of `allowed`); callers may come from several host threads.
void allow_lds(const void *kern, int bytes, std::atomic<uint64_t> &allowed) {
    int dev = 0;
    const uint64_t bit = hipGetDevice(&dev) == hipSuccess ? 1ull << (dev & 63) : 0;
    if (bit && (allowed.load(std::memory_order_acquire) & bit)) return;
    if (hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess) allowed.fetch_or(bit, std::memory_order_release);
}

// GELU (erf form) whose error is relative: gelu(v) = max(v, 0) - |v| Phi(-|v|), Phi(-t) = exp(-t^2 / 2) R(t), and R is a polynomial of degree 8 without a constant in w = 1 / (1 + 0.3 t), fitted
// to 9.2e-8 of it on 0 <= t <= 13.5 (1 / t beyond, as R has it).  128 channels share a scale that follows the largest of them, so a group whose gates all lie in the tail is held with all its
// bits: gelu_erf_h16, whose bound is absolute, is off by 0.6% at -5 and 8% at -6 there, a step of the grid.  Evaluated in float32: 1.4e-6 down to -5, 8e-6 to -13, what the exponent is rounded by; below,
// where Phi is under 2^-126, zero.  The minimum with 16 keeps |v| Phi of +inf from being inf * 0; a NaN stays one.  The block with 16384 x 1024, 2816 hidden 146 -> 148 us, 300 x 1408, 3841 hidden 25.2 both.
__device__ __forceinline__ float gelu_tail(float v) {
    const float t = fabsf(__builtin_elementwise_minimum(v, 16.f));
    const float w = __builtin_amdgcn_rcpf(fmaf(0.3f, t, 1.f));
    float p = fmaf(0.0359241813f, w, -0.158233225f);
    p = fmaf(p, w, 0.208106712f);
    p = fmaf(p, w, -0.0552709624f);
    p = fmaf(p, w, 0.129383847f);
    p = fmaf(p, w, 0.0996707305f);
    p = fmaf(p, w, 0.120791711f);
    p = fmaf(p, w, 0.119626909f);
    return fmaf(-t * (p * w), __builtin_amdgcn_exp2f(-0.72134752f * t * t), fmaxf(v, 0.f));
}

// Activations of the gated block, on float32 sums that are rounded to 4 bits of mantissa afterwards, relative to the largest of 128.
__device__ __forceinline__ float gate_of(float g, int act) {
    if (act) return gelu_tail(g);
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g));
}

// Results of a tile lie in LDS as float32, ROWS rows of COLS + 8 (rows four apart begin half the banks apart: what the two halves of a wave write).
constexpr int pitch_of(int cols) { return cols + 8; }

// To memory, eight consecutive columns a lane: stores of 16 or 32 bytes in whole rows.  The tile begins at (m0, n0).  What the results are added to is requested all at
// once: in turn with the stores each would be a trip to memory (24982 x 1024 x 316 into the stream 74 -> 54 us).
template <typename OutT, int ROWS, int COLS, int THREADS> __device__ __forceinline__ void store_tile(const LinearF8 &a, const float *park, int m0, int n0, int tid) {
    typedef OutT v8 __attribute__((ext_vector_type(8), aligned(sizeof(OutT))));
    constexpr int STEP = THREADS / (COLS / 8), IT = ROWS / STEP;
    const int N = a.w.n_rows, M = a.x.n_rows, r0 = tid / (COLS / 8), c = tid % (COLS / 8) * 8, left = N - n0 - c;
    if (left <= 0) return;
    OutT *out = (OutT *)a.c + (int64_t)(m0 + r0) * a.c_stride + n0 + c;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = a.bias && e < left ? a.bias[n0 + c + e] : 0.f;
    v8 old[sizeof(OutT) == 4 ? IT : 1];
    const bool add = sizeof(OutT) == 4 && a.accumulate;
    if (add) {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            if (m0 + r0 + i * STEP >= M) continue;
            const OutT *p = out + (int64_t)(i * STEP) * a.c_stride;
            if (left >= 8) old[sizeof(OutT) == 4 ? i : 0] = *reinterpret_cast<const v8 *>(p);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) old[sizeof(OutT) == 4 ? i : 0][e] = p[e];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (m0 + r0 + i * STEP >= M) continue;
        OutT *p = out + (int64_t)(i * STEP) * a.c_stride;
        v8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = park[(r0 + i * STEP) * pitch_of(COLS) + c + e] + bias[e];
            if (add) v += to_f32(old[sizeof(OutT) == 4 ? i : 0][e]);
            o[e] = from_f32<OutT>(v);
        }
        if (left >= 8) *reinterpret_cast<v8 *>(p) = o;
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) p[e] = o[e];
        }
    }
}

// act(gate) * up as float32 rows: 32 columns of the gate and 32 of `up` take turns in the tile, whose first hidden channel is n0.
template <int ROWS, int COLS> __device__ __forceinline__ void store_gated(float *h, int64_t stride, int M, int F, int act, const float *park, int m0, int n0, int tid, int threads) {
    for (int p = tid; p < ROWS * (COLS / 8); p += threads) {
        const int r = p / (COLS / 8), c = (p % (COLS / 8)) * 4, left = F - n0 - c;
        if (m0 + r >= M || left <= 0) continue;
        const float *at = park + r * pitch_of(COLS) + (c / 32) * 64 + c % 32;
        const f32x4 gate = *reinterpret_cast<const f32x4 *>(at), up = *reinterpret_cast<const f32x4 *>(at + 32);
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = e < left ? gate_of(gate[e], act) * up[e] : 0.f;
        *reinterpret_cast<f32x4 *>(h + (m0 + r) * stride + n0 + c) = y;      // rows are padded to four channels
    }
}

// The same held in 8 bits; the tile has whole groups of 128 hidden channels, 16 neighbouring lanes to a group of a row.
template <int ROWS, int COLS> __device__ __forceinline__ void hold_gated(const F8Rows &h, int act, const float *park, int m0, int n0, int tid, int threads) {
    static_assert(COLS == 2 * kF8Group, "");
    for (int p = tid; p < ROWS * (COLS / 16); p += threads) {
        const int r = p / (COLS / 16), c = p % (COLS / 16) * 8;
        if (m0 + r >= h.n_rows) continue;                          // whole groups leave
        const float *at = park + r * pitch_of(COLS) + (c / 32) * 64 + c % 32;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = n0 + c + e < h.width ? gate_of(at[e], act) * at[32 + e] : 0.f;
        f8_hold8(h, m0 + r, n0 + c, y);
    }
}

// What a kernel works on: C (a.c) or, of the gated block, the hidden rows: in 8 bits, or as float32 in `loose` on the way there.
struct TileArgs {
    LinearF8 a;
    F8Rows hidden;
    float *loose;
    int64_t loose_stride;
    int act, tiles_n, n_tiles;
};

// Tiles of BM rows by BN outputs, k-tiles of 128 in a ring of ST stages that LDS-direct loads fill up to ST - 1 k-tiles ahead, four waves of BM/2 x
// BN/2; a stage holds rows of 128 bytes, chunk c of row r in slot c ^ swz(r), which puts the rows of a 16-lane pass of a read on different banks.
// The scales of four k-tiles, a dword a row, come the same way into one of two places; of a dword in a register the lowest byte is the
// present k-tile's.  GATED: 32 rows of the gate and the 32 of `up` for the same hidden channels take turns in the tile.
// KS parts of k, four waves and a ring each, whose sums meet at the end: where no CU has a second workgroup, what a k-tile takes is one wave's reads, barrier and
// products in turn, and two such chains run beside each other.
// What bounds it with one tile a CU is that chain, about 0.4 us a k-tile of 128 x 128 (the sizes at launch_tiles); 9945 x 1027 x 4096 in float32, 702 tiles on 512 places,
// takes 99 us with the matrix unit busy 37% of it, 4096^3 with full rounds 1057 TFLOP/s of the bfloat16 instruction's 1270 in a library product.
// HELD: a tile of 256 has whole groups of 128 hidden channels and holds them in 8 bits itself.
template <int BM, int BN, int ST, int KS, typename OutT, bool GATED, bool EXACT, bool HELD>
__global__ __launch_bounds__(256 * KS) void f8_ring_kernel(TileArgs t) {
    constexpr int MI = BM / 64, NI = BN / 64;
    constexpr int LA = BM / 32, LB = BN / 32, LPW = LA + LB;   // 1 KB loads (8 rows x 128 bytes) per wave and k-tile
    constexpr int STB = (BM + BN) * 128, NS = (BM + BN) / 64;  // bytes of a stage; 256-byte loads of scales
    constexpr int PART = ST * STB + 2 * (BM + BN) * 4;         // bytes of a part's ring and scales
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_all[];

    const int per = (t.n_tiles + 7) >> 3;                      // workgroups congruent mod 8 share an XCD: a contiguous run of tiles for each
    const int tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if (tile >= t.n_tiles) return;
    const F8Rows &x = t.a.x, &w = t.a.w;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, part = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 8);
    unsigned char *lds = lds_all + part * PART;
    const int l32 = lane & 31, g = lane >> 5;
    const int tm = tile / t.tiles_n, tn = tile - tm * t.tiles_n;
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);
    const int wm = wave >> 1, wn = wave & 1;
    const int KT = x.groups(), steps = (KT + KS - 1) / KS, k0 = part * steps;      // this part's k-tiles: k0 .. k0 + steps - 1, as far as there are
    const int N = GATED ? w.n_rows / 2 : w.n_rows, last_m = x.n_rows - 1 - m0, last_n = N - 1 - n0;   // rows past the end: the last one again, never stored

    const int lr = lane >> 3, lc0 = (lane & 7) ^ ((lr >> 1) & 3);
    uint32_t a_off[LA], b_off[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int blk = wave * LA + i;
        a_off[i] = (uint32_t)min(blk * 8 + lr, last_m) * (uint32_t)x.code_stride + (uint32_t)((lc0 ^ (((blk >> 1) & 1) << 2)) * 16);
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int blk = wave * LB + i;
        const int row = GATED ? (blk >> 3) * 32 + (blk & 3) * 8 + lr : blk * 8 + lr;
        b_off[i] = (uint32_t)min(row, last_n) * (uint32_t)w.code_stride + (uint32_t)((lc0 ^ (((blk >> 1) & 1) << 2)) * 16);
    }
    const uint8_t *a_base = x.codes + m0 * x.code_stride, *b_base = w.codes + n0 * w.code_stride;
    const int64_t up = GATED ? (int64_t)N * w.code_stride : 0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)SJD_F8_LPTR(lds);
    // load q of this wave for this part's k-tile kt; past the end the last k-tile again, into a stage that is not read any more
    auto request1 = [&](int kt, int stage, int q) {
        const uint32_t st = lds0 + (uint32_t)(stage * STB);
        const int64_t k = (int64_t)min(k0 + kt, KT - 1) * 128;
        if (q < LA) dma16(a_base + k, a_off[q < LA ? q : 0], st + (uint32_t)((wave * LA + q) * 1024));
        else {
            const int i = q < LA ? 0 : q - LA;
            dma16(b_base + k + (((wave * LB + i) >> 2) & 1 ? up : 0), b_off[i], st + (uint32_t)(BM * 128 + (wave * LB + i) * 1024));
        }
    };
    // the scales of k-tiles 4 group ..: 64 rows a load
    auto request_scales = [&](int group) {
        if (group * 4 >= KT) return;
#pragma unroll
        for (int o = 0; o < NS; o += 4) {
            const int q = o + wave;
            if (q < NS) {
                const uint32_t to = lds0 + (uint32_t)(ST * STB + (group & 1) * (BM + BN) * 4 + q * 256);
                if (q < BM / 64) dma4(x.scales + m0 * x.scale_stride + 4 * group, (uint32_t)min(q * 64 + lane, last_m) * (uint32_t)x.scale_stride, to);
                else {
                    const int r = (q - BM / 64) * 64 + lane;
                    const uint32_t row = GATED ? (uint32_t)min((r >> 6) * 32 + l32, last_n) + (uint32_t)((r >> 5) & 1) * (uint32_t)N : (uint32_t)min(r, last_n);
                    dma4(w.scales + n0 * w.scale_stride + 4 * group, row * (uint32_t)w.scale_stride, to);
                }
            }
        }
    };
    uint32_t sa[MI], sb[NI];
    auto read_scales = [&](int group, uint32_t (&a)[MI], uint32_t (&b)[NI]) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(lds + ST * STB + (group & 1) * (BM + BN) * 4);
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = p[(wm * MI + i) * 32 + l32];
#pragma unroll
        for (int j = 0; j < NI; ++j) b[j] = p[BM + (wn * NI + j) * 32 + l32];
    };
    struct Frags { i32x4 a[2][MI], b[2][NI]; };                // half a k-tile: 64 k, of which a lane has 16 and 16
    const int swz = ((l32 >> 1) & 3) | (((l32 >> 4) & 1) << 2);
    auto read = [&](Frags &f, int stage, int half) {
        const unsigned char *st = lds + stage * STB;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int o = l32 * 128 + (((2 * (2 * half + ks) + g) ^ swz) << 4);
#pragma unroll
            for (int i = 0; i < MI; ++i) f.a[ks][i] = *reinterpret_cast<const i32x4 *>(st + (wm * MI + i) * 4096 + o);
#pragma unroll
            for (int j = 0; j < NI; ++j) f.b[ks][j] = *reinterpret_cast<const i32x4 *>(st + BM * 128 + (wn * NI + j) * 4096 + o);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    // The products of half a k-tile, and between them loads q0 .. of k-tile kt: requested in one go they hold the wave up until the
    // address unit has taken them all.
    constexpr int HALF = LPW / 2, NM = MI * NI;
    auto multiply = [&](const Frags &f, int kt, int stage, int q0) {
        Half2 wb[2][EXACT ? NI : 1];
        if constexpr (EXACT) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) wb[ks][j] = widen(f.b[ks][j], f8_scale(sb[j] & 255));
        }
        int m = 0;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            Half2 wa[2];
            if constexpr (EXACT) {
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) wa[ks] = widen(f.a[ks][i], f8_scale(sa[i] & 255));
            }
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if constexpr (EXACT) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j] = Half16<bf16>::mfma(wa[q >> 1].v[q & 1], wb[q >> 1][j].v[q & 1], acc[i][j]);
                } else {
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(f.a[0][i], f.a[1][i]), join(f.b[0][j], f.b[1][j]), acc[i][j], 0, 0, 0,
                                                                                (int)sa[i], 0, (int)sb[j]);
                }
                const int lo = m * HALF / NM, hi = (m + 1) * HALF / NM;
                if (hi > lo) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int q = 0; q < HALF; ++q)
                        if (q >= lo && q < hi) request1(kt, stage, q0 + q);
                    __builtin_amdgcn_sched_barrier(0);
                }
                ++m;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // This wave's part of the next k-tile has landed (younger ones may be on their way; scales that came before it have landed too) and its reads of this one
    // are done; then everyone's, and nobody reads this k-tile's stage any more.
    auto next_tile = [&]() {
        wait_loads<(ST - 2) * LPW>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    request_scales(k0 / 4);
    request_scales(k0 / 4 + 1);
#pragma unroll
    for (int s = 0; s < ST - 1; ++s)
#pragma unroll
        for (int q = 0; q < LPW; ++q) request1(s, s, q);
    next_tile();
#pragma unroll
    for (int q = 0; q < HALF; ++q) request1(ST - 1, ST - 1, q);
    Frags f0, f1;
    read(f0, 0, 0);
    read_scales(k0 / 4, sa, sb);
    if constexpr (KS > 1) {
#pragma unroll
        for (int i = 0; i < MI; ++i) sa[i] >>= 8 * (k0 & 3);
#pragma unroll
        for (int j = 0; j < NI; ++j) sb[j] >>= 8 * (k0 & 3);
    }
    int stage = 0, prev = ST - 1;
    for (int kt = 0; kt < steps; ++kt) {
        if (KS > 1 && k0 + kt >= KT) {                         // the last part has fewer: it only keeps the others company at the barrier
            __builtin_amdgcn_s_barrier();
            continue;
        }
        // The other place held the scales before these, last read before the barrier that ended k-tile kt - 1; they are read at the end of k-tile kt + 3,
        // after a wait for loads that are requested after these (of k-tile kt + 4, ST <= 5).
        if (((k0 + kt) & 3) == 0 && kt) request_scales((k0 + kt) / 4 + 1);
        read(f1, stage, 1);
        multiply(f0, kt + ST - 1, prev, HALF);
        next_tile();
        prev = stage;
        stage = stage + 1 == ST ? 0 : stage + 1;
        read(f0, stage, 0);
        multiply(f1, kt + ST, prev, 0);
        if (((k0 + kt) & 3) == 3) read_scales((k0 + kt) / 4 + 1, sa, sb);    // past the last k-tile: of no use to anyone
        else {
#pragma unroll
            for (int i = 0; i < MI; ++i) sa[i] >>= 8;
#pragma unroll
            for (int j = 0; j < NI; ++j) sb[j] >>= 8;
        }
    }
    static_assert(ST >= 2 && ST <= 5, "");
    __builtin_amdgcn_s_waitcnt(0);            // all loads have landed and all reads are done before LDS is reused
    __syncthreads();
    float *park = reinterpret_cast<float *>(lds_all);
#pragma unroll
    for (int q = KS - 1; q >= 0; --q) {                        // the sums of the last part, then of the one before added, ..
        if (KS == 1 || part == q) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        float &p = park[((wm * MI + i) * 32 + 8 * (v >> 2) + 4 * g + (v & 3)) * pitch_of(BN) + (wn * NI + j) * 32 + l32];
                        p = q == KS - 1 ? acc[i][j][v] : acc[i][j][v] + p;
                    }
        }
        __syncthreads();
    }
    if constexpr (HELD) hold_gated<BM, BN>(t.hidden, t.act, park, m0, n0, tid, 256 * KS);
    else if constexpr (GATED) store_gated<BM, BN>(t.loose, t.loose_stride, x.n_rows, N, t.act, park, m0, n0, tid, 256 * KS);
    else store_tile<OutT, BM, BN, 256 * KS>(t.a, park, m0, n0, tid);
}

template <int BM, int BN, int ST, int KS, typename OutT, bool GATED, bool EXACT, bool HELD = false> void launch_ring(TileArgs t, hipStream_t s) {
    constexpr int cols = GATED ? BN / 2 : BN;
    const int outs = GATED ? t.a.w.n_rows / 2 : t.a.w.n_rows;
    t.tiles_n = (outs + cols - 1) / cols;
    t.n_tiles = (t.a.x.n_rows + BM - 1) / BM * t.tiles_n;
    constexpr int stages = KS * (ST * (BM + BN) * 128 + 2 * (BM + BN) * 4), park = BM * pitch_of(BN) * 4, smem = stages > park ? stages : park;
    static_assert(smem <= 160 * 1024, "");
    auto kern = f8_ring_kernel<BM, BN, ST, KS, OutT, GATED, EXACT, HELD>;
    static std::atomic<uint64_t> allowed{0};
    allow_lds(reinterpret_cast<const void *>(kern), smem, allowed);
    kern<<<(t.n_tiles + 7) / 8 * 8, 256 * KS, smem, s>>>(t);
}


// ------------------------------------------------------------------------------------------------
// Launches that fill the chip, 16-bit results and the gated block: one workgroup of eight waves per CU stays and walks over tiles of 256 x 256,
// each wave 128 x 64 of them.  A k-tile of 128 is a whole 128-byte line of every row; 128 rows of it are a unit of 16 KB, a k-tile four units (two of the
// left operand, two of the right), and nine units form a ring: while k-tile t is multiplied, t + 1 and the first unit of t + 2 land, and the stream of requests
// runs on into the next tile.  The scales of four k-tiles, a dword a row, take turns in two places behind the ring.
// The weight is the left operand of the instruction, so that a lane's registers are one row's outputs, four consecutive ones at a time: halves of a wave swap
// registers and hold sixteen bytes each, and results go to memory without LDS; of the gated block a row's largest is mostly found in a lane.
// us in a row of calls: 8192^3 406 to 439 by card, 2500 to 2710 TFLOP/s, bound by power (1.8 GHz, the matrix unit busy 72% of the cycles); 32768 x 4096 x 1024 130, bound by its 268 MB of results, which leave
// all CUs at once (112 without the stores); 16384 x 1024 with 2816 hidden channels 97 and 44 under the profiler, the gate's activations on the vector unit.  Two workgroups of 128 x 128 tiles of
// the kernel above read each operand twice as often.
constexpr int W_UNITS = 9, W_UNIT = 16 * 1024, W_SCALES = W_UNITS * W_UNIT, W_MORE = W_SCALES + 2 * 512 * 4;
constexpr int W_LDS = W_MORE + 256 * 16;         // behind the scales: two tiles' bias (1 KB each), or the four waves' largest of each row
constexpr int W_CB = 4;                          // column tiles per column block of the tile order
constexpr int kOutside = 0x7FFFFFF0;             // a lane offset past any buffer range this kernel declares
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef int i32x2 __attribute__((ext_vector_type(2)));
// A buffer of wave-uniform base and size, said to be so: one in vector registers costs a loop at every access.
__device__ __forceinline__ rsrc_t uniform_buffer(const void *base, int bytes) {
    const uint64_t p = (uint64_t)base;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)p), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// KIND: of the gated block the activation; else how results are stored: W_WHOLE rows of whole 16-byte pieces, W_PAST the same past the caches, W_ANY rows that
// begin and end anywhere.
constexpr int W_WHOLE = 0, W_PAST = 1, W_ANY = 2;
template <typename OutT, bool GATED, int KIND> __global__ __launch_bounds__(512) void f8_wide_kernel(TileArgs t, int tiles_m) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const F8Rows &x = t.a.x, &w = t.a.w;
    const int tiles_n = t.tiles_n, KT = x.groups();
    constexpr int COLS = GATED ? 128 : 256;
    const int M = x.n_rows, N = GATED ? w.n_rows / 2 : w.n_rows;

    // Workgroups congruent mod 8 share an XCD: each XCD owns a run of row panels and walks it column block by column block, row by row inside a block,
    // so that the weight rows of a block stay in its L2 while the row panels stream past.
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, n_slots = gridDim.x >> 3;
    const int rp0 = (int)((long long)xcd * tiles_m / 8), nrp = (int)((long long)(xcd + 1) * tiles_m / 8) - rp0;
    const int n_mine = nrp * tiles_n;
    auto tile_of = [&](int li) {
        if (li >= n_mine) return -1;
        const int cb = li / (nrp * W_CB);
        const int left = tiles_n - cb * W_CB, cbw = left < W_CB ? left : W_CB;
        const int lo = li - cb * nrp * W_CB;
        const int r = lo / cbw;
        return (rp0 + r) * tiles_n + cb * W_CB + (lo - r * cbw);
    };
    int li = slot;
    int tile = tile_of(li);
    if (tile < 0) return;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int wm = wave >> 2, wn = wave & 3;

    // Of every unit a wave brings the rows 16 wave .., two loads of eight rows (1 KB); chunk c of row r goes to slot c ^ swz(r), swz(r) = bits 1, 2 and 4 of r.
    // GATED: 32 rows of the gate and the 32 of `up` for the same channels take turns, so a wave's rows are of one of them.
    const int lr = lane >> 3;
    const uint32_t chunk = (uint32_t)(((lane & 7) ^ ((lr >> 1) & 3) ^ ((wave & 1) << 2)) * 16);
    const uint32_t a_lane = lr * (uint32_t)x.code_stride + chunk, b_lane = lr * (uint32_t)w.code_stride + chunk;
    // Of each operand the bytes from a tile's first row to the end of the last one there is: rows past it are outside of what the descriptor holds and come as zeros.
    struct Src { rsrc_t a, b; };
    auto make_src = [&](int tl) {
        const int tm = tl / tiles_n, tn = tl - tm * tiles_n;
        const int rows = min(M - tm * 256, 256), outs = min(N - tn * COLS, COLS);
        Src s;
        s.a = __builtin_amdgcn_make_buffer_rsrc(x.codes + (int64_t)tm * 256 * x.code_stride, 0, (rows - 1) * (int)x.code_stride + KT * 128, 0x00020000);
        s.b = __builtin_amdgcn_make_buffer_rsrc(w.codes + ((int64_t)tn * COLS + (GATED && ((wave >> 1) & 1) ? N : 0)) * w.code_stride, 0, (outs - 1) * (int)w.code_stride + KT * 128, 0x00020000);
        return s;
    };
    const uint32_t lds0 = (uint32_t)(uintptr_t)SJD_F8_LPTR(lds);
    // load q (0..3 left, 4..7 right operand; two to a unit) of k-tile kt, whose first unit is `unit`
    auto up = [](int u, int d) { u += d; return u >= W_UNITS ? u - W_UNITS : u; };
    auto issue = [&](const Src &s, int kt, int unit, int q) {
        const uint32_t to = lds0 + (uint32_t)(up(unit, q >> 1) * W_UNIT + wave * 2048 + (q & 1) * 1024);
        const int u = (q >> 1) & 1, r = wave * 16 + (q & 1) * 8;
        const uint32_t off = q < 4 ? a_lane + (uint32_t)(u * 128 + r) * (uint32_t)x.code_stride
                                   : b_lane + (uint32_t)(GATED ? (u * 2 + (wave >> 2)) * 32 + (r & 31) : u * 128 + r) * (uint32_t)w.code_stride;
        // one wait state, for M0: five for the descriptor would cost 3% of 8192^3, and the compiler keeps it in scalar registers (the built kernels are checked for it)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(q < 4 ? s.a : s.b), "s"(kt * 128) : "memory");
    };
    // The scales of k-tiles 4 group .. of tile tl: 64 rows a wave, the left operand's first.
    auto issue_scales = [&](int tl, int group, int place) {
        int lane;                                                   // counted anew: what a tile keeps for the next one is a register too many
        asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
        const int tm = tl / tiles_n, tn = tl - tm * tiles_n;
        const uint32_t to = lds0 + (uint32_t)(W_SCALES + place * 2048 + wave * 256);
        if (wave < 4) dma4(x.scales + (int64_t)tm * 256 * x.scale_stride + 4 * group, (uint32_t)min(wave * 64 + lane, M - 1 - tm * 256) * (uint32_t)x.scale_stride, to);
        else {
            const int row = GATED ? min(tn * 128 + (wave - 4) * 32 + (lane & 31), N - 1) + (lane >> 5) * N : min(tn * 256 + (wave - 4) * 64 + lane, N - 1);
            dma4(w.scales + 4 * group, (uint32_t)row * (uint32_t)w.scale_stride, to);
        }
    };
    int sc[6], sn[6];                            // of the four row groups and the two column groups: this k-tile's and the next one's
    auto read_scales = [&](int place, int byte) {
        const unsigned char *p = lds + W_SCALES + place * 2048 + byte + l32 * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) sn[i] = p[(wm * 4 + i) * 128];
#pragma unroll
        for (int j = 0; j < 2; ++j) sn[4 + j] = p[1024 + (wn * 2 + j) * 128];
    };

    const int swz = ((l32 >> 1) & 3) | (((l32 >> 4) & 1) << 2);
    int fk[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) fk[c] = l32 * 128 + (((2 * c + g) ^ swz) << 4);
    i32x8 fa[4], fb[2][2];
    auto read = [&](const unsigned char *at, int ks) {
        return join(*reinterpret_cast<const i32x4 *>(at + fk[2 * ks]), *reinterpret_cast<const i32x4 *>(at + fk[2 * ks + 1]));
    };
    // the fragments of half ks of the k-tile whose first unit is `unit`
    auto read_a = [&](int unit, int ks, int i) { fa[i] = read(lds + up(unit, wm) * W_UNIT + i * 4096, ks); };
    auto read_b = [&](int unit, int ks, int j) { fb[ks][j] = read(lds + up(unit, 2 + (wn >> 1)) * W_UNIT + (wn & 1) * 8192 + j * 4096, ks); };
    // Sums begin with the bias, which waits in LDS: the next tile's 256 of it come while a tile is multiplied.  Without one the two places hold zeros.
    f32x16 acc[4][2];
    auto issue_bias = [&](int tl, int at) {                     // columns past the end: the last one's
        if (!GATED && t.a.bias && wave < 4)
            dma4(t.a.bias, (uint32_t)min((tl % tiles_n) * 256 + wave * 64 + lane, N - 1) * 4u, lds0 + (uint32_t)(W_MORE + at * 1024 + wave * 256));
    };
    auto begin = [&](int at) {
        const float *bias = reinterpret_cast<const float *>(lds + W_MORE + at * 1024) + wn * 64 + 4 * g;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 b = {0.f, 0.f, 0.f, 0.f};
                if constexpr (!GATED) b = *reinterpret_cast<const f32x4 *>(bias + 32 * j + 8 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = b[e];
            }
    };

    // One k-tile: sixteen matrix instructions of this wave, each a slot with its LDS reads and loads pinned.  Its operands are units h .. h + 3 (mod 9), those
    // of the next one h + 4 .. h + 7.  The first unit of the one after goes to h + 8 in the first half.  After the second slot of the second half, when
    // all of this k-tile's fragments are in registers: wait until this wave's loads of the next k-tile have landed (the two younger ones may stay in
    // flight), then the barrier; the rest reads the next k-tile's scales and first fragments and requests the other units of the one after into h, h + 1, h + 2.
    auto ktile = [&](auto younger, int h, const Src &rs, int r_kt, int place, int byte) {
        const int h1 = up(h, 4), h2 = up(h, 8);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const bool last = ks == 1;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const int i = m >> 1, j = m & 1;
                if (!last && m == 0) { read_b(h, 1, 0); read_b(h, 1, 1); }
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[ks][j], fa[i], acc[i][j], 0, 0, 0, sc[4 + j], 0, sc[i]);
                __builtin_amdgcn_sched_barrier(0);
                if (last && m == 1) {
                    wait_loads<2 + decltype(younger)::value>();
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    read_b(h1, 0, 0);
                    read_b(h1, 0, 1);
                    read_scales(place, byte);
                }
                if (last && m >= 2) issue(rs, r_kt, h2, m);
                if (!last && (m == 2 || m == 5)) issue(rs, r_kt, h2, m == 5);
                if (j == 1) read_a(last ? h1 : h, last ? 0 : 1, i);      // row group i is done for this half: fetch the next one's
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int i = 0; i < 6; ++i) sc[i] = sn[i];
    };

    issue_scales(tile, 0, 0);
    issue_bias(tile, 0);
    if (!GATED && !t.a.bias && tid < 128) *reinterpret_cast<f32x4 *>(lds + W_MORE + tid * 16) = f32x4{0.f, 0.f, 0.f, 0.f};
    Src rs = make_src(tile);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int q = 0; q < 8; ++q) issue(rs, s, 4 * s, q);
    __builtin_amdgcn_s_waitcnt(0x0070);       // both k-tiles, scales and bias have landed
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) read_a(0, 0, i);
    read_b(0, 0, 0);
    read_b(0, 0, 1);
    read_scales(0, 0);
#pragma unroll
    for (int i = 0; i < 6; ++i) sc[i] = sn[i];
    begin(0);
    int h = 0, place = 0, bias_at = 0;

    while (true) {
        const int tm = tile / tiles_n, tn = tile - tm * tiles_n;
        li += n_slots;
        const int tile_next = tile_of(li);
        const int tile_req = tile_next >= 0 ? tile_next : tile;      // no next tile: this one's first k-tiles again (in bounds, never used)
        bias_at ^= 1;
        issue_bias(tile_req, bias_at);
        auto step = [&](auto younger, int kt) {
            if (kt + 2 == KT) rs = make_src(tile_req);
            // the place of the scales before these, which every wave has read; they land before the wait of this k-tile
            if ((kt & 3) == 0) issue_scales(kt + 4 < KT ? tile : tile_req, kt + 4 < KT ? kt / 4 + 1 : 0, place ^ 1);
            const bool turn = (kt & 3) == 3 || kt + 1 == KT;
            if (turn) place ^= 1;
            ktile(younger, h, rs, kt + 2 >= KT ? kt + 2 - KT : kt + 2, place, turn ? 0 : (kt & 3) + 1);
            h = up(h, 4);
        };
        // the last tile's stores are younger than the loads that the first k-tile waits for: four at least, or sixteen
        step(std::integral_constant<int, GATED ? 4 : 16>(), 0);
        for (int kt = 1; kt < KT; ++kt) step(std::integral_constant<int, 0>(), kt);
        // Here the next tile's first k-tile is in LDS and the second on its way.  Register 4 q + e of a lane is output 8 q + 4 g + e of row l32 of a block.
        // What lies outside the result falls outside the buffer descriptor.
        const int row0 = tm * 256 + wm * 128, rows_left = min(max(M - row0, 0), 128);
        if constexpr (GATED) {
            const int col0 = tn * 128 + wn * 32;
            uint8_t *hbase = t.hidden.codes + (int64_t)row0 * t.hidden.code_stride + tn * 128;
            const int pitch = (int)t.hidden.code_stride;
            const rsrc_t h_rs = uniform_buffer(hbase, rows_left ? (rows_left - 1) * pitch + 128 : 0);
            uint8_t *sbase = t.hidden.scales + (int64_t)row0 * t.hidden.scale_stride + tn;
            const int s_pitch = (int)t.hidden.scale_stride;
            const rsrc_t s_rs = uniform_buffer(sbase, rows_left ? (rows_left - 1) * s_pitch + 1 : 0);
            float *largest = reinterpret_cast<float *>(lds + W_MORE) + wm * 512;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][0][v] = gate_of(acc[i][0][v], KIND) * acc[i][1][v];
                if (col0 + 32 > N) {                              // hidden channels that are not there
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (col0 + 8 * (v >> 2) + 4 * g + (v & 3) >= N) acc[i][0][v] = 0.f;
                }
                float top = 0.f;                                  // the maximum passes over NaN
#pragma unroll
                for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(acc[i][0][v]));
                if (__builtin_amdgcn_ballot_w64(top == INFINITY)) {
                    uint32_t fine = 0;
#pragma unroll
                    for (int v = 0; v < 16; ++v) fine = max(fine, f8_finite_mag(acc[i][0][v]));
                    top = __uint_as_float(fine);
                }
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                largest[(i * 32 + l32) * 4 + wn] = top;
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 m = *reinterpret_cast<const f32x4 *>(largest + (i * 32 + l32) * 4);
                const uint32_t byte = f8_scale_byte(__float_as_uint(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]))));
                uint32_t c[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    typedef short s16x2 __attribute__((ext_vector_type(2)));
                    s16x2 p = {0, 0};
                    p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, acc[i][0][4 * q], acc[i][0][4 * q + 1], f8_scale(byte), false);
                    p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, acc[i][0][4 * q + 2], acc[i][0][4 * q + 3], f8_scale(byte), true);
                    c[q] = __builtin_bit_cast(uint32_t, p);
                }
                // the lower lanes take both halves' registers 0 and 1 (channels 0 .. 15), the upper ones 2 and 3
                const auto s0 = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false), s1 = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
                const i32x4 out = {(int)s0[0], (int)s0[1], (int)s1[0], (int)s1[1]};
                const int r = i * 32 + l32;
                __builtin_amdgcn_raw_buffer_store_b128(out, h_rs, r < rows_left ? r * pitch + wn * 32 + g * 16 : kOutside, 0, 0);
                hold_stored(out);
                if (wn == 0) __builtin_amdgcn_raw_buffer_store_b8((uint8_t)byte, s_rs, r < rows_left && !g ? r * s_pitch : kOutside, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const int col0 = tn * 256 + wn * 64, cols_left = N - col0;
            const int pitch = (int)t.a.c_stride * (int)sizeof(OutT);
            OutT *cbase = (OutT *)t.a.c + (int64_t)row0 * t.a.c_stride + col0;
            const rsrc_t c_rs = uniform_buffer(cbase, rows_left && cols_left > 0 ? (rows_left - 1) * pitch + min(cols_left, 64) * (int)sizeof(OutT) : 0);
            // Sixteen rows of 128 bytes at a time through the wave's part of the free unit, which it refills itself, and out in whole lines.  Chunk c of row r lies
            // in slot c ^ (r / 2): the sixteen rows of a write, and the two of a sixteen-lane pass of a read, on different banks.
            unsigned char *park = lds + up(h, 8) * W_UNIT + wave * 2048;
            const int l16 = l32 & 15, w_at = l16 * 128 + 8 * g, w_swz = l16 >> 1;
            const int rr = lane >> 3, rc = lane & 7;
            int lane_off = rc * 8 < cols_left ? rr * pitch + rc * 16 : kOutside;
            asm volatile("" : "+v"(lane_off));        // or the row offsets of a tile move out of the tile loop into registers it does not have
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                i32x2 o[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        typedef OutT v4 __attribute__((ext_vector_type(4)));
                        v4 p;
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e] = from_f32<OutT>(acc[i][j][4 * q + e]);
                        o[j][q] = __builtin_bit_cast(i32x2, p);
                    }
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    if ((l32 >> 4) == hh) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int q = 0; q < 4; ++q) *reinterpret_cast<i32x2 *>(park + w_at + (((4 * j + q) ^ w_swz) << 4)) = o[j][q];
                    }
                    asm volatile("" ::: "memory");       // a wave's LDS operations execute in order: no wait, only the order
                    __builtin_amdgcn_wave_barrier();
                    if constexpr (KIND == W_ANY) {               // a row a store, a column a lane
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const uint16_t o = *reinterpret_cast<const uint16_t *>(park + r * 128 + ((rr ^ (r >> 1)) << 4) + rc * 2);
                            const int r0 = i * 32 + hh * 16 + r;
                            __builtin_amdgcn_raw_buffer_store_b16(o, c_rs, r0 < rows_left && lane < cols_left ? lane * 2 : kOutside, r0 * pitch, 0);
                        }
                        asm volatile("" ::: "memory");
                        __builtin_amdgcn_wave_barrier();
                    } else {
                        i32x4 out[2];
#pragma unroll
                        for (int p = 0; p < 2; ++p) out[p] = *reinterpret_cast<const i32x4 *>(park + (p * 8 + rr) * 128 + ((rc ^ ((p * 8 + rr) >> 1)) << 4));
                        asm volatile("" ::: "memory");
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const int r0 = i * 32 + hh * 16 + p * 8;
                            __builtin_amdgcn_raw_buffer_store_b128(out[p], c_rs, r0 + rr < rows_left ? lane_off : kOutside, r0 * pitch, KIND == W_PAST ? 2 : 0);
                            hold_stored(out[p]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);       // lgkmcnt(0): this wave has read back what it parked
        }
        if (tile_next < 0) break;
        begin(bias_at);
        tile = tile_next;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);       // the loads of the unused last requests have landed before the LDS goes away
}

// ------------------------------------------------------------------------------------------------
// Few tiles: 32 rows by 32 outputs (gated: 16 hidden channels) a workgroup, the k-tiles dealt to its four waves.  A wave has a ring of ST k-tiles of its own
// (64 rows of 128 bytes and their scales, 8 KB and a line each), fills it with LDS-direct loads and waits for nobody; the four sums meet at the end.
// What bounds it is what one CU gets from memory, about 64 KB a microsecond after three microseconds of launch and first trip, so the tile is small:
// 17 rows by 1024 outputs of 4096 take 6.0 us, with 64x64 tiles 10.3; one row of 4096 by 1024 outputs 4.2 us.
template <int ST, typename OutT, bool GATED, bool EXACT> __global__ __launch_bounds__(256) void f8_thin_kernel(TileArgs t) {
    constexpr int STB = 64 * 128 + 256, LOADS = 9, P = 40;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_all[];
    const LinearF8 &a = t.a;
    const F8Rows &x = a.x, &w = a.w;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, g = lane >> 5, lr = lane >> 3;
    const int COLS = GATED ? 16 : 32, N = GATED ? w.n_rows / 2 : w.n_rows, M = x.n_rows;
    const int n0 = blockIdx.x * COLS, m0 = blockIdx.y * 32, KT = x.groups();
    unsigned char *lds = lds_all + wave * (ST * STB);
    const uint32_t lds0 = (uint32_t)(uintptr_t)SJD_F8_LPTR(lds);
    const uint8_t *a_base = x.codes + m0 * x.code_stride, *b_base = w.codes + n0 * w.code_stride, *u_base = GATED ? b_base + (int64_t)N * w.code_stride : b_base;
    uint32_t off[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const int r = (q & 3) * 8 + lr;                        // rows past the end: the last one again, never stored
        const uint32_t row = q < 4 ? (uint32_t)min(r, M - 1 - m0) * (uint32_t)x.code_stride : (uint32_t)min(GATED ? r & 15 : r, N - 1 - n0) * (uint32_t)w.code_stride;
        off[q] = row + (uint32_t)(((lane & 7) ^ ((lr >> 1) & 3) ^ (((q >> 1) & 1) << 2)) * 16);
    }
    const uint8_t *scale = g ? w.scales + (int64_t)(n0 + min(GATED ? l32 & 15 : l32, N - 1 - n0) + (GATED && l32 >= 16 ? N : 0)) * w.scale_stride
                             : x.scales + (int64_t)(m0 + min(l32, M - 1 - m0)) * x.scale_stride;
    auto request = [&](int i, int stage) {                     // this wave's k-tile i, past the end the last one again
        const int kt = min(wave + 4 * i, KT - 1);
        const uint32_t to = lds0 + (uint32_t)(stage * STB);
        const int64_t k = (int64_t)kt * 128;
#pragma unroll
        for (int q = 0; q < 8; ++q) dma16((q < 4 ? a_base : GATED && q >= 6 ? u_base : b_base) + k, off[q], to + q * 1024);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(to + 8192), "v"(scale + (kt >> 2) * 4) : "memory");
    };
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    const int swz = ((l32 >> 1) & 3) | (((l32 >> 4) & 1) << 2);
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) request(s, s);
    int stage = 0;
    for (int i = 0; wave + 4 * i < KT; ++i) {
        wait_loads<(ST - 2) * LOADS>();                        // this k-tile has landed, and the reads of the one before are done
        __builtin_amdgcn_sched_barrier(0);
        const unsigned char *st = lds + stage * STB;
        i32x4 fa[4], fb[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int o = l32 * 128 + (((2 * c + g) ^ swz) << 4);
            fa[c] = *reinterpret_cast<const i32x4 *>(st + o);
            fb[c] = *reinterpret_cast<const i32x4 *>(st + 4096 + o);
        }
        const uint32_t sa = *reinterpret_cast<const uint32_t *>(st + 8192 + l32 * 4) >> (8 * wave), sb = *reinterpret_cast<const uint32_t *>(st + 8320 + l32 * 4) >> (8 * wave);
        __builtin_amdgcn_sched_barrier(0);
        request(i + ST - 1, stage == 0 ? ST - 1 : stage - 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (EXACT) {
#pragma unroll
                for (int c = 2 * h; c < 2 * h + 2; ++c) {
                    const Half2 p = widen(fa[c], f8_scale(sa & 255)), q = widen(fb[c], f8_scale(sb & 255));
                    acc = Half16<bf16>::mfma(p.v[0], q.v[0], acc);
                    acc = Half16<bf16>::mfma(p.v[1], q.v[1], acc);
                }
            } else {
                acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(fa[2 * h], fa[2 * h + 1]), join(fb[2 * h], fb[2 * h + 1]), acc, 0, 0, 0, (int)sa, 0, (int)sb);
            }
        }
        stage = stage + 1 == ST ? 0 : stage + 1;
    }
    __builtin_amdgcn_s_waitcnt(0);                             // the last requests have landed before the ring is parked over
    __builtin_amdgcn_sched_barrier(0);
    constexpr int PARK = ST * STB / 4;
    float *park = reinterpret_cast<float *>(lds_all);          // [wave] at its ring: 32 rows of P floats
#pragma unroll
    for (int v = 0; v < 16; ++v) park[wave * PARK + (8 * (v >> 2) + 4 * g + (v & 3)) * P + l32] = acc[v];
    __syncthreads();
    const int r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 4;
    auto sum = [&](int col) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(park + r * P + col);
#pragma unroll
        for (int o = 1; o < 4; ++o) v += *reinterpret_cast<const f32x4 *>(park + o * PARK + r * P + col);
        return v;
    };
    const int left = N - n0 - c;
    if (m0 + r >= M || left <= 0 || c >= COLS) return;
    const f32x4 v = sum(c);
    if constexpr (GATED) {
        const f32x4 u = sum(16 + c);
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = e < left ? gate_of(v[e], t.act) * u[e] : 0.f;
        *reinterpret_cast<f32x4 *>(t.loose + (m0 + r) * t.loose_stride + n0 + c) = y;
    } else {
        OutT *out = (OutT *)a.c + (int64_t)(m0 + r) * a.c_stride + n0 + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) {
                float y = v[e];
                if (a.bias) y += a.bias[n0 + c + e];
                if (sizeof(OutT) == 4 && a.accumulate) y += to_f32(out[e]);
                out[e] = from_f32<OutT>(y);
            }
    }
}

template <int ST, typename OutT, bool GATED, bool EXACT> void launch_thin(const TileArgs &t, hipStream_t s) {
    constexpr int cols = GATED ? 16 : 32, smem = 4 * ST * (64 * 128 + 256);
    const int outs = GATED ? t.a.w.n_rows / 2 : t.a.w.n_rows;
    auto kern = f8_thin_kernel<ST, OutT, GATED, EXACT>;
    static std::atomic<uint64_t> allowed{0};
    allow_lds(reinterpret_cast<const void *>(kern), smem, allowed);
    kern<<<dim3((outs + cols - 1) / cols, (t.a.x.n_rows + 31) / 32), 256, smem, s>>>(t);
}

// ------------------------------------------------------------------------------------------------
// The gate for few rows and short k in one launch: 32 rows by 128 hidden channels, which is one scale, a workgroup; each of its eight waves has the 32 weight rows
// of 16 channels (gate, then up) in a ring of its own, the rows of x are shared.  A launch less than tiles that leave float32 behind for norm_f8.hip to hold; for k
// beyond 1024 its 288 bytes of a k from memory take one CU longer than those two launches.  What bounds it is those bytes, at 50 KB a microsecond.  The whole block, us in a graph / in calls with
// kept operands / with operands wrapped anew, two launches -> this: 64 x 256, 2816 hidden 11.1 / 14.1 / 17.1 -> 10.2 / 11.3 / 14.2; 64 x 512, 1300 10.2 / 13.9 / 17.2 -> 10.4 / 11.4 / 14.3; 1 x 512, 2816
// 10.1 / 13.7 / 17.3 -> 10.6 / 11.3 / 14.0; one row of 1024, 2816 11.3 / 13.7 / 17.2 -> 13.2 / 13.1 / 14.4; 64 x 1024, 2816 13.2 / 14.3 / 17.0 -> 14.1 / 13.9 / 14.2; 200 x 1024, 2816 18.0 / 18.0 / 18.3 ->
// 15.0 / 14.6 / 14.8; 300 x 1024, 2816 20.0 / 19.6 / 19.9 -> 17.4 / 17.1 / 17.1.  Calls outside of a graph, which wait for the host, are as short or shorter everywhere; in a graph it wins with k up to 256, from 64 workgroups
// with 512 and from 88 with 1024, and with fewer it loses, 1.33 times at the most (1 x 1024, 256 hidden 8.2 -> 10.9).  One rule for both: a captured call has the bits and the workspace of an eager one.
template <int ST> __global__ __launch_bounds__(512) void f8_gate_kernel(TileArgs t) {
    constexpr int STB = (32 + 256) * 128, SCALES = ST * STB, LARGEST = SCALES + 2 * 8 * 256;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const F8Rows &x = t.a.x, &w = t.a.w;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, g = lane >> 5, lr = lane >> 3;
    const int M = x.n_rows, F = w.n_rows / 2, KT = x.groups();
    const int n0 = blockIdx.x * 128, c0 = n0 + wave * 16, m0 = blockIdx.y * 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)SJD_F8_LPTR(lds);
    // rows past the end: the last one again, never stored
    const int first = min(c0, F - 1);                             // a wave may have no channels at all
    const uint8_t *a_base = x.codes + m0 * x.code_stride, *b_base = w.codes + first * w.code_stride, *u_base = b_base + F * w.code_stride;
    auto chunk = [&](int q) { return (uint32_t)(((lane & 7) ^ ((lr >> 1) & 3) ^ (((q >> 1) & 1) << 2)) * 16); };
    const uint32_t a_off = (uint32_t)min((wave & 3) * 8 + lr, M - 1 - m0) * (uint32_t)x.code_stride + chunk(wave & 3);
    uint32_t b_off[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) b_off[q] = (uint32_t)min((q & 1) * 8 + lr, F - 1 - first) * (uint32_t)w.code_stride + chunk(q);
    const uint8_t *scale = g ? w.scales + ((int64_t)first + min(l32 & 15, F - 1 - first) + (l32 >= 16 ? F : 0)) * w.scale_stride
                             : x.scales + (int64_t)(m0 + min(l32, M - 1 - m0)) * x.scale_stride;
    auto request = [&](int kt, int stage) {                       // past the end the last k-tile again
        const uint32_t to = lds0 + (uint32_t)(stage * STB);
        const int64_t k = (int64_t)min(kt, KT - 1) * 128;
        if (wave < 4) dma16(a_base + k, a_off, to + wave * 1024);
#pragma unroll
        for (int q = 0; q < 4; ++q) dma16((q < 2 ? b_base : u_base) + k, b_off[q], to + 4096 + wave * 4096 + q * 1024);
    };
    auto request_scales = [&](int group) {
        if (group * 4 >= KT) return;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(lds0 + (uint32_t)(SCALES + (group & 1) * 2048 + wave * 256)), "v"(scale + group * 4) : "memory");
    };
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    const int swz = ((l32 >> 1) & 3) | (((l32 >> 4) & 1) << 2);
    request_scales(0);
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) request(s, s);
    int stage = 0;
    for (int kt = 0; kt < KT; ++kt) {
        wait_loads<(ST - 2) * 4>();                              // this wave's part of the k-tile has landed, and its reads of the one before are done
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const unsigned char *st = lds + stage * STB, *sc = lds + SCALES + ((kt >> 2) & 1) * 2048 + wave * 256 + (kt & 3);
        i32x4 fa[4], fb[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int o = l32 * 128 + (((2 * c + g) ^ swz) << 4);
            fa[c] = *reinterpret_cast<const i32x4 *>(st + o);
            fb[c] = *reinterpret_cast<const i32x4 *>(st + 4096 + wave * 4096 + o);
        }
        const uint32_t sa = sc[l32 * 4], sb = sc[128 + l32 * 4];
        __builtin_amdgcn_sched_barrier(0);
        if ((kt & 3) == 0) request_scales(kt / 4 + 1);           // read four k-tiles from here, behind waits for loads that are requested later
        request(kt + ST - 1, stage == 0 ? ST - 1 : stage - 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 4; ++c) {                            // the weight on the left: a lane's registers are one row's channels
            const Half2 p = widen(fb[c], f8_scale(sb)), q = widen(fa[c], f8_scale(sa));
            acc = Half16<bf16>::mfma(p.v[0], q.v[0], acc);
            acc = Half16<bf16>::mfma(p.v[1], q.v[1], acc);
        }
        stage = stage + 1 == ST ? 0 : stage + 1;
    }
    // register 4 q + e is channel 8 q + 4 g + e of row l32, of the gate for q < 2, else of `up`
    float y[8];
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        y[v] = c0 + 8 * (v >> 2) + 4 * g + (v & 3) < F ? gate_of(acc[v], t.act) * acc[8 + v] : 0.f;
        top = max(top, f8_finite_mag(y[v]));
    }
    const auto both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    uint32_t *largest = reinterpret_cast<uint32_t *>(lds + LARGEST);
    if (!g) largest[l32 * 8 + wave] = max(both[0], both[1]);
    __builtin_amdgcn_s_waitcnt(0);                               // the last requests have landed too
    __syncthreads();
#pragma unroll
    for (int o = 0; o < 8; ++o) top = max(top, largest[l32 * 8 + o]);
    const uint32_t byte = f8_scale_byte(top);
    const uint2 c = f8_encode8(y, byte);
    // the lower lanes take channels 0 .. 7 of their row, the upper ones 8 .. 15
    const auto s = __builtin_amdgcn_permlane32_swap(c.x, c.y, false, false);
    if (m0 + l32 < M) {
        *reinterpret_cast<uint2 *>(t.hidden.codes + (int64_t)(m0 + l32) * t.hidden.code_stride + c0 + 8 * g) = uint2{s[0], s[1]};
        if (wave == 0 && !g) t.hidden.scales[(int64_t)(m0 + l32) * t.hidden.scale_stride + blockIdx.x] = (uint8_t)byte;
    }
}

void launch_gate(const TileArgs &t, hipStream_t s) {
    constexpr int ST = 4, smem = ST * (32 + 256) * 128 + 2 * 8 * 256 + 32 * 8 * 4;
    static_assert(smem <= 160 * 1024, "");
    auto kern = f8_gate_kernel<ST>;
    static std::atomic<uint64_t> allowed{0};
    allow_lds(reinterpret_cast<const void *>(kern), smem, allowed);
    kern<<<dim3((t.a.w.n_rows / 2 + 127) / 128, (t.a.x.n_rows + 31) / 32), 512, smem, s>>>(t);
}

int device_cus() {
    static std::atomic<int> cus{0};
    int c = cus.load(std::memory_order_acquire);
    if (c == 0) {
        int dev = 0;
        hipDeviceProp_t prop;
        c = (hipGetDevice(&dev) == hipSuccess && hipGetDeviceProperties(&prop, dev) == hipSuccess) ? prop.multiProcessorCount : 256;
        if (c < 8) c = 8;
        cus.store(c, std::memory_order_release);
    }
    return c;
}

template <typename OutT, bool GATED, int KIND> void launch_wide(TileArgs t, hipStream_t s) {
    constexpr int cols = GATED ? 128 : 256;
    const int outs = GATED ? t.a.w.n_rows / 2 : t.a.w.n_rows, tiles_m = (t.a.x.n_rows + 255) / 256;
    t.tiles_n = (outs + cols - 1) / cols;
    const int per_xcd = ((tiles_m + 7) / 8) * t.tiles_n;      // tiles of the XCD with the most row panels
    const int slots = per_xcd < device_cus() / 8 ? per_xcd : device_cus() / 8;
    auto kern = f8_wide_kernel<OutT, GATED, KIND>;
    static std::atomic<uint64_t> allowed{0};
    allow_lds(reinterpret_cast<const void *>(kern), W_LDS, allowed);
    kern<<<8 * slots, 512, W_LDS, s>>>(t, tiles_m);
}

// Results of more than half of what the last-level cache holds go past the caches: they push the weights out of it and are gone before they are read.  us alone /
// with a call that reads them, through the caches -> past them: 32768 x 4096 x 1024 144 / 220 -> 136 / 220, 8192^3 400 / 450 -> 393 / 447; with 64 MB,
// 8192 x 4096 x 4096, 110 / 125 -> 108 / 128.
template <typename OutT> void launch_wide_rows(const TileArgs &t, hipStream_t s) {
    const LinearF8 &a = t.a;
    if (a.w.n_rows % 8 || a.c_stride % 8 || (uintptr_t)a.c % 16) launch_wide<OutT, false, W_ANY>(t, s);
    else if ((int64_t)a.x.n_rows * a.w.n_rows * 2 >= 128ll << 20) launch_wide<OutT, false, W_PAST>(t, s);
    else launch_wide<OutT, false, W_WHOLE>(t, s);
}

// Two k-tiles at least, since requests run two ahead into the next tile but no further; offsets inside a tile of results in 32 bits.
bool wide_takes(const LinearF8 &a) { return a.dtype != 0 && a.x.width > kF8Group && a.c_stride * 2 * 128 < (1ll << 31); }

int64_t tiles(int64_t rows, int64_t outs, int bm, int bn) { return (rows + bm - 1) / bm * ((outs + bn - 1) / bn); }

// Whatever is not for the persistent kernel, by the 256 CUs of this chip: the smallest tile of which no CU has more than one (two of the smallest), or two or three with a shorter ring where that
// fills more of the chip than the next larger tile; at last two workgroups with 128x128 tiles to a CU.  A tile of half the size reads more of both operands, but time is what one CU gets through while it walks k.  us, M x N x K, the weight from memory, as thin / 64x64 /
// 128x64 / 128x128 with one workgroup to a CU / with two: 64 x 1024 x 2816 5.1 / 8.5 / 11.2 / 15.6 / 22.3; 16 x 8192 x 8192 17.4 / 22.8 / 26.3 / 41.8 / 76.0;
// 512 x 1024 x 4096 9.9 / 11.1 / 15.1 / 21.0 / 31.4; 256 x 2304 x 768 6.1 / 5.6 / 6.3 / 8.2 / 9.7; 1024 x 1024 x 4096 - / 11.6 / 15.2 / 21.1 / 31.5; 512 x 4096 x 1024 - / 11.4 / 7.7 / 9.6 / 12.0;
// 2048 x 1024 x 4096 - / 20.9 / 16.1 / 21.5 / 31.6; 1024 x 4096 x 1024 - / 18.9 / 13.0 / 11.3 / 13.6; 2048 x 4096 x 1024 - / - / 22.9 / 20.0 / 16.3.
// Several to a CU, 128x128 one / two / 64x64 three / 128x64 two / three: 700 x 2900 x 1408 13.0 / 16.4 / 10.1 / 12.4 / 13.7 (up to two 64x64 tiles a CU); 900 x 2900 x 1408 13.3 / 16.8 / 12.7 /
// 13.1 / 14.1, 300 x 6900 x 1408 13.0 / 16.6 / 13.7 / 12.7 / 13.8 (up to one and a half 128x64 tiles a CU); with 256 tiles of 128x128, 2048^3, 16.5 / 21.1 / 21.1 / 17.4 / 18.7; 3000 x 1500 x 2048
// 29.0 / 22.3 / 21.9 / 23.2 / 19.5 and 1024 x 5632 x 4096 51.4 / 47.0 / 57.7 / 47.9 / 43.8 (up to three 128x64 tiles a CU).  Exact products alike: 700 x 2900 x 1408 17.7 / 20.2 / 15.5 / 16.9 /
// 18.3, 3000 x 1500 x 2048 40.4 / 32.6 / 31.7 / 33.1 / 30.3; the gated block with 700 x 1408, 2816 hidden 28.2 / 22.5 / 22.2 / 23.4 / 20.3.
template <typename OutT, bool GATED, bool EXACT> void launch_tiles(const TileArgs &t, hipStream_t s) {
    const int64_t M = t.a.x.n_rows, N = t.a.w.n_rows;
    constexpr int64_t kCus = 256;
    if constexpr (!GATED || EXACT) {                              // few tiles of the gate sum exact products (launch_gated_f8)
        if (tiles(M, N, 32, 32) <= kCus) return launch_thin<3, OutT, GATED, EXACT>(t, s);
        if (tiles(M, N, 32, 32) <= 2 * kCus) return launch_thin<2, OutT, GATED, EXACT>(t, s);
    }
    if (tiles(M, N, 64, 64) <= kCus) launch_ring<64, 64, 3, 2, OutT, GATED, EXACT>(t, s);
    else if (tiles(M, N, 128, 64) <= kCus) launch_ring<128, 64, 4, 1, OutT, GATED, EXACT>(t, s);
    else if (tiles(M, N, 64, 64) <= 2 * kCus) launch_ring<64, 64, 3, 1, OutT, GATED, EXACT>(t, s);
    else if (tiles(M, N, 128, 64) <= kCus * 3 / 2) launch_ring<128, 64, 3, 1, OutT, GATED, EXACT>(t, s);
    else if (tiles(M, N, 128, 128) <= kCus) launch_ring<128, 128, 3, 1, OutT, GATED, EXACT>(t, s);
    else if (tiles(M, N, 128, 64) <= 3 * kCus) launch_ring<128, 64, 2, 1, OutT, GATED, EXACT>(t, s);
    else launch_ring<128, 128, 2, 1, OutT, GATED, EXACT>(t, s);
}

}  // namespace

void launch_linear_f8(const LinearF8 &a, hipStream_t s) {
    const TileArgs t{a, {}, nullptr, 0, 0, 0, 0};
    if (wide_takes(a) && f8_wide_before_tiles(a.x.n_rows, a.w.n_rows)) {
        if (a.dtype == 1) launch_wide_rows<bf16>(t, s);
        else launch_wide_rows<f16>(t, s);
    } else if (a.dtype == 0) launch_tiles<float, false, true>(t, s);
    else if (a.dtype == 1) launch_tiles<bf16, false, false>(t, s);
    else launch_tiles<f16, false, false>(t, s);
}

// Which launch holds the hidden rows in 8 bits itself: it has whole groups of 128 channels.
static bool gate_in_one(const F8Rows &x, const F8Rows &w) { return x.width <= 1024 && tiles(x.n_rows, w.n_rows, 32, 256) <= 256; }
static bool gate_fills(const F8Rows &x, const F8Rows &w) { return x.width > kF8Group && f8_gate_fills(x.n_rows, w.n_rows / 2); }
bool gated_f8_holds(const F8Rows &x, const F8Rows &w, int dtype) { return gate_in_one(x, w) || (dtype != 0 && gate_fills(x, w)); }

void launch_gated_f8(const GatedF8 &g, hipStream_t s) {
    LinearF8 a{};
    a.x = g.x;
    a.w = g.w;
    const TileArgs t{a, g.hidden, g.loose, g.loose_stride, g.act, 0, 0};
    if (gate_in_one(g.x, g.w)) return launch_gate(t, s);
    // A hidden value next to a border of the 8-bit grid goes to either side with what the 8-bit instruction drops, a step of 1/16 to 1/8 away: 1.6e-3 of the results over
    // many values, but one of a few hundred may be half a percent.  bfloat16 results are rounded by as much (1.7e-3), half ones by 2e-4: theirs, as float32 ones, sum exact products.
    // Few tiles wait for memory and sum exact products in the same time (64 x 5632 x 1024 5.3 us and 5.4); tiles that multiply take a quarter as long
    // again (300 x 7682 x 1408 with the norms' launch 16.0 and 19.9), and where the chip is full the block takes twice as long or more: 16384 x 1024, 2816 hidden 135 and 317, 4096 x 1024, 2816 52 and 97.
    if (g.dtype == 1 && gate_fills(g.x, g.w)) return g.act ? launch_wide<float, true, 1>(t, s) : launch_wide<float, true, 0>(t, s);
    if (g.dtype == 2 && gate_fills(g.x, g.w)) return launch_ring<128, 256, 3, 1, float, true, true, true>(t, s);
    if (g.dtype != 1 || tiles(a.x.n_rows, a.w.n_rows, 32, 32) <= 512) launch_tiles<float, true, true>(t, s);
    else launch_tiles<float, true, false>(t, s);
    NormF8 n{};
    n.x = g.loose; n.x_stride = g.loose_stride; n.out = g.hidden;
    launch_norm_f8<float>(n, false, s);
}

}  // namespace sjd
