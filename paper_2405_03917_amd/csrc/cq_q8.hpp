// Declarations of the 8-bit block cache (cq_*_q8): formats, arguments of its kernels, and how its bytes stand for numbers.
#pragma once

#include "cq_internal.hpp"

namespace cq {

constexpr int kQ8Head = 128;                                // channels of a head
constexpr int kQ8TileBytes = kTileTokens * kQ8Head;         // of keys [token][channel] or of values [channel][token]
constexpr int kQ8Pairs = kQ8Head / 2;
constexpr int kQ8RowTiles = 256;                           // most tiles of a piece of the context where a KV head has few rows
constexpr int kQ8Partial = kQ8Head + kPartialHeader;        // floats of a partial row: reference, sum, channels

struct Q8Cache {
    uint8_t* codes[2];                                      // keys, values
    float* scales[2];                                       // one per tile, in the order of the tiles
    CacheMap map;
};

// Token row j of a call with m rows of sequence n sits at position t_n - m + j; rows in front of position 0 are padding.
struct Q8Rows {
    int batch, m, t, n_kv_heads;
    const int32_t* seq_lens;
    __device__ __forceinline__ int length(int n) const { return seq_lens ? min(max(seq_lens[n], 0), t) : t; }
};

struct Q8AppendArgs : Q8Rows {
    const uint16_t* x[2];                                   // keys, values: fp16 [batch][m][n_kv_heads][128] by strides
    int64_t x_batch_stride, x_row_stride;
    Q8Cache cache;
    const double2* tile_tab;                                // cos, sin of 64 tile theta_i: [tile][pair] (null: no rotation)
    const double2* lane_tab;                                // cos, sin of u theta_i: in the order of lane_entry
    const uint16_t* q;                                      // queries to rotate (null: none), by strides
    int64_t q_batch_stride, q_row_stride;
    int n_q_heads;
    uint16_t* q_out;                                        // fp16 [batch][m][n_q_heads][128]
    // set by the launcher
    int slots;                                              // tiles of a sequence that rows of the call can lie in
    int heads, q_heads;                                     // heads in a row that a workgroup (a thread, of queries) takes
    unsigned kv_wgs;                                        // workgroups of keys, and of values
};
cq_status launch_append_q8(const Q8AppendArgs& a, int kind, hipStream_t stream);
size_t q8_rope_table_bytes(int positions);
cq_status launch_q8_rope_table(double base, int positions, void* table, hipStream_t stream);

struct Q8DequantArgs : Q8Rows {
    Q8Cache cache;
    uint16_t* out[2];                                       // keys, values (null: not wanted): fp16 [batch][m][n_kv_heads][128] by strides
    int64_t out_batch_stride, out_row_stride;
    int slots;
    unsigned kv_wgs;
};
cq_status launch_dequantize_q8(const Q8DequantArgs& a, int kind, hipStream_t stream);

struct Q8AttentionArgs : Q8Rows {
    const uint16_t* q;                                      // fp16 [batch][m][n_q_heads][128]
    uint16_t* out;
    Q8Cache cache;
    float scale_log2e;
    int n_q_heads;
    int tiles_per_split, n_split;
    float* partials;                                        // [batch][m][n_q_heads][n_split][kQ8Partial]
    int row_block;                                          // rows of a KV head that a workgroup serves
    unsigned* counters;                                     // arrivals per (stream, row block); null: merge_q8_kernel follows

    // Tiles that the rows of a block look at, and how many pieces of the context have any (one at least: it writes the rows of
    // sequences of no tokens).  A row block of one piece goes to the output at once.
    __device__ __forceinline__ int block_tiles(int t_n, int block) const
    {
        const int qper = n_q_heads / n_kv_heads, last = (min((block + 1) * row_block, m * qper) - 1) / qper;
        return max((t_n - m + last + kTileTokens) / kTileTokens, 0);
    }
    __device__ __forceinline__ int pieces(int n_tiles) const { return max((n_tiles - 1) / tiles_per_split + 1, 1); }
};
// How a call is cut: which kernel, tiles per split.  A function of the sizes alone.
struct Q8Plan {
    int row_block;                                          // rows of a KV head that a workgroup serves
    int tiles_per_split, n_split;
};
Q8Plan q8_plan(int batch, int n_kv_heads, int n_q_heads, int m, int t, int tokens_per_split);
// Many rows per KV head (cq_q8_chunk.hip): 128 or 256 of them to a workgroup.
cq_status launch_chunk_q8(const Q8AttentionArgs& a, int kind, int row_block, hipStream_t stream);
cq_status launch_attention_q8(const Q8AttentionArgs& a, int kind, const Q8Plan& plan, hipStream_t stream);

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 q8_half8 __attribute__((ext_vector_type(8)));
typedef float q8_float4 __attribute__((ext_vector_type(4)));
typedef unsigned q8_u4 __attribute__((ext_vector_type(4)));

// Four code bytes as fp16 numbers, exactly.  An integer c is the byte c + 128, and 0x6400 + byte is the fp16 number 1024 + byte: a
// byte permute for two of them and one packed addition.  e4m3: the conversion instruction.
template <int KIND>
__device__ __forceinline__ void q8_halves(unsigned w, half2_t* lo, half2_t* hi)
{
    if constexpr (KIND == CQ_Q8_INT8) {
        const half2_t bias = {(_Float16)-1152.f, (_Float16)-1152.f};
        *lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + bias;
        *hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + bias;
    } else {
        *lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
        *hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
    }
}
template <int KIND>
__device__ __forceinline__ q8_half8 q8_half8_of(unsigned w0, unsigned w1)
{
    half2_t a, b, c, d;
    q8_halves<KIND>(w0, &a, &b);
    q8_halves<KIND>(w1, &c, &d);
    return q8_half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr float kQ8Lowest = -3.402823466e38f;
// Weights are 2^(score - reference + kQ8Above) with a reference that the largest score may pass by kQ8Slack before it is moved: at most
// 2^15 in fp16, and those of 2^-14 of fp16's normal numbers are 2^-21 of the largest, its smallest 2^-31.
constexpr float kQ8Slack = 8.f, kQ8Above = 7.f;

// The bytes of tokens that are not there (from `from` on, of 16 in order) become zero: an e4m3 byte may be no number, and its
// weight of zero would not hide it.
__device__ __forceinline__ q8_u4 q8_only_before(q8_u4 w, int from)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int keep = from - 4 * i;
        w[i] = keep >= 4 ? w[i] : keep <= 0 ? 0u : w[i] & (0xffffffffu >> (32 - 8 * keep));
    }
    return w;
}
#endif

}  // namespace cq
