// A key/value cache held in 4 bits, and the norms and rotation of queries and keys in front of it: layout, conversions, launchers.
//
// A page holds 64 tokens; each head has 68 * dim bytes of it in one piece, a "block".  NG = dim / 32 groups of 32 channels share a
// power of two (the byte e + 127, 255: not a number), a value is a 4-bit float (two exponent bits, one mantissa bit: 0, 1/2, 1, 3/2, 2,
// 3, 4, 6 and their negatives) times that power - what gfx950 converts in one instruction for two values, exactly, since two
// significant bits fit every type it converts to.
//
// Inside a block everything lies as the lanes of the 16x16x32 matrix instruction want it, 16 tokens (a subtile) at a time:
//   keys    [token][dim / 2 bytes]: lane t + 16 j takes the NG dwords j NG .. of token t, so that the NG instructions of a subtile
//           run over all channels and a subtile is one contiguous load of 4 NG bytes a lane
//   values  [subtile][lane n + 16 j][4 tokens 4 j ..][NG]: the byte holds channels 32 g + 2 n and the next one of a token, so that
//           a lane's dwords hold, for its four tokens, one channel pair of every group; again one contiguous load a subtile
//   key scales    [t][g][subtile]: one dword a lane and group for the four subtiles
//   value scales  [j][subtile][token][g]
#pragma once
#include "common.h"

namespace sjd {

constexpr int kKv4Page = 64;
__host__ __device__ constexpr size_t kv4_block_bytes(int dim) { return (size_t)68 * dim; }

__host__ __device__ __forceinline__ uint32_t kv4_k_code(int dim, int off, int chunk8) { return off * (dim / 2) + chunk8 * 4; }      // 8 channels
__host__ __device__ __forceinline__ uint32_t kv4_v_code(int dim, int off, int n) {                                        // NG bytes, channels 32 g + 2 n, + 1
    return 32 * dim + (off >> 4) * 8 * dim + ((((off & 15) >> 2) * 16 + n) * 4 + (off & 3)) * (dim / 32);
}
__host__ __device__ __forceinline__ uint32_t kv4_k_scale(int dim, int off, int g) { return 64 * dim + ((off & 15) * (dim / 32) + g) * 4 + (off >> 4); }
__host__ __device__ __forceinline__ uint32_t kv4_v_scale(int dim, int off) {                                              // NG bytes
    return 66 * dim + ((((off & 15) >> 2) * 4 + (off >> 4)) * 4 + (off & 3)) * (dim / 32);
}

struct Kv4Cache {
    uint8_t *pages;
    int n_pages, n_heads, dim;
};

// Norms and rotation of sjd_qk_opts, checked.
struct QkOpts {
    int norm;                       // 0 none, 1 x / sqrt(mean x^2 + eps) * gain, 2 (x - mean) / sqrt(var + eps) * gain + shift
    float eps;
    const float *q_gain, *q_shift, *k_gain, *k_shift;   // [dim], nullptr: 1, 0
    int rot, adjacent, n_axes;      // the first `rot` channels turn: (i, i + rot/2) or (2i, 2i + 1)
    int axis_end[4];                // pair i belongs to the first axis a with i < axis_end[a]
    const float *freq;              // [rot / 2]
};

struct QkRows {
    const void *q, *k, *v;          // rows; heads follow one another
    int64_t q_stride, k_stride, v_stride;      // elements
    void *q_out, *k_out;
    int64_t q_out_stride, k_out_stride;
    const int32_t *pos;             // [n_rows, n_axes]
    const int32_t *slot;            // [n_rows]: page * 64 + offset
    int n_rows, n_heads, n_kv, dim;
};

// out = rotate(norm(rows)) for queries and keys (each nullable)
template <typename T> void launch_qk_rope(const QkOpts &o, const QkRows &r, hipStream_t s);
// keys and values into the cache; o != nullptr: the keys normed and rotated first (and queries, where given, to q_out)
template <typename T> void launch_kv4_write(const Kv4Cache &c, const QkOpts *o, const QkRows &r, hipStream_t s);
template <typename T> void launch_kv4_read(const Kv4Cache &c, const int32_t *slot, void *k, int64_t k_stride, void *v, int64_t v_stride,
                                           int n_rows, hipStream_t s);

struct Kv4Attn {
    Kv4Cache cache;
    const void *q;
    void *o;
    int64_t q_stride, o_stride;
    const int32_t *q_start, *kv_len, *table;   // q_start nullable: max_q rows each
    int64_t table_stride;
    int n_seqs, n_heads, n_rows, max_pages, max_q, max_kv;
    int causal, skip, window;
    float scale_log2;
    int tile, n_tiles;              // rows of a workgroup, workgroups over the rows of a sequence and key head
    int z0;                         // the first of n_tiles * n_splits that a launch takes
    int group;                      // query heads of a key head
    uint32_t group_magic;           // row / group = row * group_magic >> 32 (0: a group of one)
    int n_splits, split_pages;      // a sequence's pages in pieces of split_pages, joined by a second launch where n_splits > 1
    float *partial, *partial_ml;    // [n_rows][n_heads][n_splits][dim] sums; [..][2] reference (times scale, base 2) and denominator
};
bool kv4_attention_plan(Kv4Attn &a, bool is_f32);              // fills tile .. group_magic, n_splits, split_pages; false: too large
size_t kv4_attention_workspace(const Kv4Attn &a);              // bytes of partial, for those
template <typename T> void launch_kv4_attention(const Kv4Attn &a, hipStream_t s);

}  // namespace sjd
