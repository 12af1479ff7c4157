// Attention over the 8-bit block cache (cq_decode_attention_q8, cq_chunk_attention_q8) for few rows per KV head, and the merge of
// context pieces, for gfx950.
//
//   s = scale k_scale (q . k_code),  p = 2^(s log2(e) - ref),  out = sum_tiles v_scale sum_i p_i v_code_i / sum_i p_i
//
// A wavefront walks whole tiles by itself, everything in registers: S^T = K Q^T and O^T = V^T P^T by 16x16x32 products, rows of the
// KV head (query heads of a token, tokens of a chunk) in the 16 columns.  The result of S^T holds, in the lane of column n
// and block g, rows 4 g + e; rows of key tile b are tokens 16 g + 4 b + e, so a lane's scores of b = 0 .. 3 are tokens 16 g .. 16 g + 15, in
// order: what the lane feeds into the second product, whose other operand (16 tokens of a channel) is 16 bytes of the cache as they lie.
// Bound by memory: 16 KB a tile against 512 products' clocks and about 1000 of conversions.
#include <algorithm>

#include "cq_q8.hpp"

namespace cq {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
// One row's weighted values from its pieces: `n` of (reference, sum, 128 channels), `stride` floats apart; channel i.
__device__ __forceinline__ float merged(const float* p, int n, size_t stride, int i)
{
    float m = kQ8Lowest, l = 0.f, o = 0.f;
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
        const float ms = p[s * stride], ls = p[s * stride + 1], os = p[s * stride + kPartialHeader + i];
        const float m_new = fmaxf(m, ms);
        const float keep = __builtin_amdgcn_exp2f(m - m_new), w = __builtin_amdgcn_exp2f(ms - m_new);
        // (a piece without tokens leaves its channels unwritten)
        l = fmaf(l, keep, ls * w);
        o = fmaf(o, keep, ls > 0.f ? os * w : 0.f);
        m = m_new;
    }
    return l > 0.f ? o / l : 0.f;
}

__global__ __launch_bounds__(kThreads) void merge_q8_kernel(const float* partials, uint16_t* out, int64_t rows, int n_split)
{
    const int64_t row = (int64_t)blockIdx.x * (kThreads / kQ8Head) + threadIdx.x / kQ8Head;
    const int i = threadIdx.x % kQ8Head;
    if (row >= rows) return;
    const _Float16 h = (_Float16)merged(partials + row * n_split * kQ8Partial, n_split, kQ8Partial, i);
    out[row * kQ8Head + i] = __builtin_bit_cast(uint16_t, h);
}

template <int KIND, int RB>
__global__ __launch_bounds__(kThreads) void rows_q8_kernel(Q8AttentionArgs a, int row_blocks, unsigned units)
{
    __shared__ float lds[kWaves][16 * RB][kQ8Partial];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    // the row blocks of a piece of a stream run on one XCD, which shares what it reads
    const unsigned eighth = blockIdx.x >> 3;
    const int block = eighth % row_blocks;
    const unsigned unit = (eighth / row_blocks) * 8 + (blockIdx.x & 7);
    if (unit >= units) return;
    const int split = unit % a.n_split, stream = unit / a.n_split;
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads;
    const int qper = a.n_q_heads / a.n_kv_heads, rows = a.m * qper, row0 = block * 16 * RB;
    const int t_n = a.length(n), pos0 = t_n - a.m;
    const int pos_first = pos0 + row0 / qper, pos_last = pos0 + (min(row0 + 16 * RB, rows) - 1) / qper;
    const int n_tiles = pos_last < 0 ? 0 : pos_last / kTileTokens + 1;
    const int tile0 = split * a.tiles_per_split, tile1 = min(tile0 + a.tiles_per_split, n_tiles);
    const float scale = fabsf(a.scale_log2e);

    int pos[RB];
    q8_half8 q[RB][4];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int row = min(row0 + 16 * r + col, rows - 1), j = row / qper;
        pos[r] = pos0 + j;
        const uint16_t* src = a.q + (((size_t)n * a.m + j) * a.n_q_heads + h * qper + (row - j * qper)) * kQ8Head;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            q[r][s] = *reinterpret_cast<const q8_half8*>(src + 64 * (s >> 1) + 16 * g + 8 * (s & 1));
            if (a.scale_log2e < 0.f) q[r][s] = -q[r][s];
        }
    }
    q8_float4 o[RB][8];
    float ref[RB], sum[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        ref[r] = kQ8Lowest;
        sum[r] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[r][c] = q8_float4{0.f, 0.f, 0.f, 0.f};
    }

    q8_u4 kr[8], vr[8];
    float ks = 0.f, vs = 0.f;
    auto request_keys = [&](size_t at) {
        const uint8_t* src = a.cache.codes[0] + at * kQ8TileBytes + (16 * (col >> 2) + (col & 3)) * kQ8Head + 16 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) kr[i] = *reinterpret_cast<const q8_u4*>(src + 4 * (i >> 1) * kQ8Head + 64 * (i & 1));
        ks = a.cache.scales[0][at];
    };
    auto request_values = [&](size_t at) {
        const uint8_t* src = a.cache.codes[1] + at * kQ8TileBytes + col * kTileTokens + 16 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) vr[i] = *reinterpret_cast<const q8_u4*>(src + 16 * i * kTileTokens);
        vs = a.cache.scales[1][at];
    };
    int tile = tile0 + wave;
    if (tile < tile1) {
        const size_t at = a.cache.map.tile_index(n, h, tile);
        request_keys(at);
        request_values(at);
    }
#pragma unroll 1
    for (; tile < tile1; tile += kWaves) {
        const bool more = tile + kWaves < tile1;
        const size_t next = a.cache.map.tile_index(n, h, more ? tile + kWaves : tile);
        q8_float4 s[RB][4];
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int b = 0; b < 4; ++b) s[r][b] = q8_float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const q8_u4 w = kr[2 * b + f];
                const q8_half8 k0 = q8_half8_of<KIND>(w[0], w[1]), k1 = q8_half8_of<KIND>(w[2], w[3]);
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    s[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[r][2 * f], s[r][b], 0, 0, 0);
                    s[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[r][2 * f + 1], s[r][b], 0, 0, 0);
                }
            }
        // (a factor of zero stands for one so small that every weight is 1: 0 times a masked -infinity is no number)
        const float by = fmaxf(scale * ks, 1e-37f);
        if (more) request_keys(next);
        const int first = tile * kTileTokens + 16 * g;
        q8_half8 p[RB][2];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            // (no fused multiply-add with the reference: a score beyond 2^24 is the rounded product, in its maximum and in its weight)
#pragma clang fp contract(off)
            float x[16], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = s[r][i >> 2][i & 3] * by;
            if (tile * kTileTokens + kTileTokens - 1 > pos_first) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = first + i > pos[r] ? -INFINITY : x[i];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
            if (__any(top > ref[r] + kQ8Slack)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float now = fmaxf(ref[r], top), keep = __builtin_amdgcn_exp2f(ref[r] - now);
                ref[r] = now;
                sum[r] *= keep;
#pragma unroll
                for (int c = 0; c < 8; ++c) o[r][c] *= keep;
            }
            const float below = ref[r] - kQ8Above;
            float w[16], part = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[i] = __builtin_amdgcn_exp2f(x[i] - below);
                part += w[i];
            }
            sum[r] += part;
#pragma unroll
            for (int i = 0; i < 16; ++i) p[r][i >> 3][i & 7] = (_Float16)w[i];
        }
        const bool cut = KIND == CQ_Q8_E4M3 && (tile + 1) * kTileTokens > t_n;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            q8_u4 w = vr[c];
            if (cut) w = q8_only_before(w, t_n - first);
            const q8_half8 v0 = q8_half8_of<KIND>(w[0], w[1]), v1 = q8_half8_of<KIND>(w[2], w[3]);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                q8_float4 y = {0.f, 0.f, 0.f, 0.f};
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[r][0], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[r][1], y, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][c][e] = fmaf(y[e], vs, o[r][c][e]);
            }
        }
        if (more) request_values(next);
    }

    // ---- the wavefronts' rows: lane (col, g) holds channels 16 c + 4 g + e of row col
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        sum[r] += __shfl_xor(sum[r], 16);
        sum[r] += __shfl_xor(sum[r], 32);
        float* dst = lds[wave][16 * r + col];
        if (g == 0) {
            dst[0] = ref[r];
            dst[1] = sum[r];
        }
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[kPartialHeader + 16 * c + 4 * g + e] = o[r][c][e];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int local = 16 * r + (tid >> 4), row = row0 + local, i0 = 8 * (tid & 15);
        if (row >= rows) continue;
        const int j = row / qper;
        const size_t at = ((size_t)n * a.m + j) * a.n_q_heads + h * qper + (row - j * qper);
        float m = kQ8Lowest, l = 0.f, y[8];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, lds[w][local][0]);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float by = __builtin_amdgcn_exp2f(lds[w][local][0] - m);
            l = fmaf(lds[w][local][1], by, l);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(lds[w][local][kPartialHeader + i0 + i], by, y[i]);
        }
        if (a.n_split == 1) {
            q8_half8 z;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = (_Float16)(l > 0.f ? y[i] / l : 0.f);
            *reinterpret_cast<q8_half8*>(a.out + at * kQ8Head + i0) = z;
        } else {
            float* dst = a.partials + (at * a.n_split + split) * kQ8Partial;
            if ((tid & 15) == 0) {
                dst[0] = m;
                dst[1] = l;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[kPartialHeader + i0 + i] = y[i];
        }
    }
}

template <int KIND>
cq_status launch_rows(const Q8AttentionArgs& a, int row_block, hipStream_t stream)
{
    const int rows = a.m * (a.n_q_heads / a.n_kv_heads), row_blocks = (rows + row_block - 1) / row_block;
    const int64_t units = (int64_t)a.batch * a.n_kv_heads * a.n_split, grid = (units + 7) / 8 * 8 * row_blocks;
    if (grid > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    if (row_block == 16) hipLaunchKernelGGL((rows_q8_kernel<KIND, 1>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a, row_blocks, (unsigned)units);
    else hipLaunchKernelGGL((rows_q8_kernel<KIND, 2>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a, row_blocks, (unsigned)units);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace

Q8Plan q8_plan(int batch, int n_kv_heads, int n_q_heads, int m, int t, int tokens_per_split)
{
    const int64_t rows = (int64_t)m * (n_q_heads / n_kv_heads);
    const int n_tiles = (t - 1) / kTileTokens + 1;
    Q8Plan p;
    // Workgroups of eight wavefronts convert a tile half as often as those of four, and reach further in front of their first row and
    // behind their last: where most of the context lies in front of the chunk.  128 -> 256 rows, us: integers, 32 heads, 512 of 16384
    // 166 -> 156, e4m3, 2 x 1024 of 8192 293 -> 271, 32 / 8 heads, 4 x 512 of 16384 568 -> 522; 2 x 4096 of 4096 348 -> 397, with 32 / 8 heads
    // 304 -> 303; 32 / 8 heads, 64 of 8192 27 -> 33.
    p.row_block = rows <= 16 ? 16 : rows <= 64 ? 32 : rows >= 512 && t - m >= 4096 ? 256 : 128;
    if (tokens_per_split) {
        p.tiles_per_split = tokens_per_split / kTileTokens;
    } else if (p.row_block > 32) {
        const int64_t blocks = (int64_t)batch * n_kv_heads * ((rows + p.row_block - 1) / p.row_block);
        const int64_t pieces = std::max<int64_t>(1, std::min<int64_t>((n_tiles + 7) / 8, 65536 / p.row_block / blocks));
        p.tiles_per_split = (int)((n_tiles + pieces - 1) / pieces);
    } else {
        const int64_t blocks = (int64_t)batch * n_kv_heads * ((rows + p.row_block - 1) / p.row_block);
        const int64_t pieces = std::max<int64_t>(1, std::min<int64_t>((n_tiles + kWaves - 1) / kWaves, 1024 / blocks));
        const int64_t tiles = (n_tiles + pieces - 1) / pieces;
        p.tiles_per_split = (int)((tiles + kWaves - 1) / kWaves * kWaves);
    }
    p.n_split = (n_tiles - 1) / p.tiles_per_split + 1;
    return p;
}

cq_status launch_attention_q8(const Q8AttentionArgs& a, int kind, const Q8Plan& plan, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.batch * a.m * a.n_q_heads, merges = (rows + kThreads / kQ8Head - 1) / (kThreads / kQ8Head);
    const cq_status st = plan.row_block > 32 ? launch_chunk_q8(a, kind, plan.row_block, stream)
                         : kind == CQ_Q8_INT8 ? launch_rows<CQ_Q8_INT8>(a, plan.row_block, stream) : launch_rows<CQ_Q8_E4M3>(a, plan.row_block, stream);
    if (st != CQ_OK || a.n_split == 1) return st;
    hipLaunchKernelGGL(merge_q8_kernel, dim3((unsigned)merges), dim3(kThreads), 0, stream, a.partials, a.out, rows, a.n_split);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace cq
