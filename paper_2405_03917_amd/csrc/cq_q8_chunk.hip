// Attention over the 8-bit block cache for many rows per KV head (cq_chunk_attention_q8), for gfx950.
//
// The products of cq_q8_attention.hip, with a tile's codes turned into fp16 once for a workgroup: its wavefronts share them through LDS
// and each serve 32 rows.  A tile lies in LDS as the operands of the products, 16 bytes a lane one behind the
// other, so that neither writing nor reading them meets a bank twice.  Two tiles' room: while one is worked off the next
// is converted, and the one after that is on its way from memory.
// Values keep their codes; a block's scale goes into its weights, relative to the accumulators' unit (2^(score - reference) by
// v_scale / unit, an addition to the exponent), and out of their sum again.  The unit moves with the scales: weights would lose bits in fp16
// under one that is far above them.
// Bound by the issue of vector and matrix instructions, which keep each other waiting: per 32 rows and tile 64 products of 16
// clocks and about 200 vector instructions, 32 exponentials among them.  Two wavefronts a SIMD that do nothing but such a mix, on
// operands from LDS, need 3450 clocks for 2048 of products; here they need 4000.  4 x 512 tokens of 16384 (e4m3, 32 / 8 heads): 515 to 521 us
// by the card, 1049 to 1038 TFLOP/s; 2 x 4096 of 4096 (integers, 32 heads): 303 to 314, 908 to 877, where tiles on the diagonal and the last
// workgroups count.  (Vector work placed between the products of its own wavefront, wavefronts half a tile apart,
// 32x32x16 products, keys straight from memory, codes in LDS: 0.95 to 0.7 of that.)
#include <algorithm>

#include "cq_q8.hpp"

namespace cq {
namespace {

constexpr int RB = 2;                                       // blocks of 16 rows of a wavefront
// Streams (pieces of them) on an XCD whose row blocks are dealt out together, the longest first: more of them end together, fewer share
// what L2 holds.  1, 2, 4, 8, all, us: integers, 32 heads, 2 x 4096 of 4096 351, 328, 320, 318, 322; 2000 of 2000 75, 75, 60, 60, 61; ragged 8 x 1024 of
// 3000 269, 260, 255, 256, 264.
constexpr unsigned kTogether = 4;
constexpr float kFaint = -3.f, kFaintest = -60.f;           // log2 of values' scales relative to the accumulators' unit, and to the largest
constexpr float kNoScale = -200.f;

template <int KIND, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void chunk_q8_kernel(Q8AttentionArgs a, int row_blocks, unsigned units)
{
    constexpr int ROWS = 16 * RB;                           // of a wavefront
    constexpr int N = 8 / WAVES;                            // 16 bytes a lane of keys, and of values, that a wavefront brings
    extern __shared__ q8_u4 lds[];                          // [2][keys, values][16 operands][64 lanes]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    // the row blocks of a piece of a stream run on one XCD, which shares what it reads; four pieces together, their longest blocks first
    const unsigned eighth = blockIdx.x >> 3, set = eighth / (kTogether * row_blocks), in_set = eighth % (kTogether * row_blocks);
    const unsigned here = min(kTogether, (units + 7) / 8 - set * kTogether);
    const int block = row_blocks - 1 - (int)(in_set / here);
    const unsigned unit = (set * kTogether + in_set % here) * 8 + (blockIdx.x & 7);
    if (unit >= units) return;
    const int split = unit % a.n_split, stream = unit / a.n_split;
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads;
    const int qper = a.n_q_heads / a.n_kv_heads, rows = a.m * qper;
    const int t_n = a.length(n), pos0 = t_n - a.m;
    const int row0 = block * (ROWS * WAVES) + wave * ROWS;
    const int n_tiles = a.block_tiles(t_n, block), pieces = a.pieces(n_tiles);
    if (split >= pieces) return;
    const int tile0 = split * a.tiles_per_split, tile1 = min(tile0 + a.tiles_per_split, n_tiles);
    // (a wavefront behind the last row repeats it and stores nothing)
    const int pos_first = pos0 + min(row0, rows - 1) / qper, pos_last = pos0 + (min(row0 + ROWS, rows) - 1) / qper;
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
    // log2 of the accumulators' unit: of a scale of the values so far, one that the tile's is between an eighth of and all of (where it is not
    // below 2^-60 of the largest so far, and makes no difference)
    float unit_log = kNoScale, largest_log = kNoScale;

    // ---- a wavefront brings N of eight parts of keys (part i: tokens b = i / 2, half i & 1 of the channels) and N of values (channel block
    // i), two operands each (as in cq_q8_attention.hip)
    q8_u4 gk[N], gv[N];
    const unsigned k_off = (16 * (col >> 2) + 4 * (wave * N >> 1) + (col & 3)) * kQ8Head + 16 * g + 64 * (wave * N & 1), v_off = (16 * N * wave + col) * kTileTokens + 16 * g;
    auto request = [&](size_t at) {
        const uint8_t* k = a.cache.codes[0] + at * kQ8TileBytes;
        const uint8_t* v = a.cache.codes[1] + at * kQ8TileBytes;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            gk[i] = *reinterpret_cast<const q8_u4*>(k + k_off + 64 * i);
            gv[i] = *reinterpret_cast<const q8_u4*>(v + v_off + 16 * i * kTileTokens);
        }
    };
    auto stage = [&](int tile, int buf) {
        q8_u4* k = lds + buf * 2048 + 128 * N * wave + lane;
        q8_u4* v = lds + buf * 2048 + 1024 + 128 * N * wave + lane;
        if (KIND == CQ_Q8_E4M3 && (tile + 1) * kTileTokens > t_n) {
#pragma unroll
            for (int i = 0; i < N; ++i) gv[i] = q8_only_before(gv[i], t_n - tile * kTileTokens - 16 * g);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            k[128 * i] = __builtin_bit_cast(q8_u4, q8_half8_of<KIND>(gk[i][0], gk[i][1]));
            k[128 * i + 64] = __builtin_bit_cast(q8_u4, q8_half8_of<KIND>(gk[i][2], gk[i][3]));
            v[128 * i] = __builtin_bit_cast(q8_u4, q8_half8_of<KIND>(gv[i][0], gv[i][1]));
            v[128 * i + 64] = __builtin_bit_cast(q8_u4, q8_half8_of<KIND>(gv[i][2], gv[i][3]));
        }
    };
    // Lane i knows where tile `known` + i lies and its scales: asked for 60 rounds at a time, since a round by itself would wait for
    // its answer (and a scalar request's, for LDS as well).
    int known = tile0;
    size_t places = 0;
    float k_scales = 0.f, v_logs = 0.f;
    auto learn = [&](int tile) {
        known = tile;
        places = a.cache.map.tile_index(n, h, min(tile + lane, tile1 - 1));
        k_scales = a.cache.scales[0][places];
        v_logs = __builtin_amdgcn_logf(a.cache.scales[1][places]);
        // (waited for here: where they are used, the requests of the next tile would be waited for as well)
        asm volatile("" : "+v"(k_scales), "+v"(v_logs));
    };
    auto place = [&](int tile) {
        const int i = tile - known;
        return (size_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)places, i) | (size_t)(unsigned)__builtin_amdgcn_readlane((int)(places >> 32), i) << 32;
    };
    auto scale_of = [&](float scales, int tile) {
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scales), tile - known));
    };
    if (tile0 < tile1) {
        learn(tile0);
        request(place(tile0));
        stage(tile0, 0);
        if (tile0 + 1 < tile1) request(place(tile0 + 1));
    }
    __syncthreads();
    int buf = 0;
#pragma unroll 1
    for (int tile = tile0; tile < tile1; ++tile, buf ^= 1) {
        if (tile - known == 60) learn(tile);
        const float ks = scale_of(k_scales, tile), v_log = scale_of(v_logs, tile);
        if (tile + 1 < tile1) {
            stage(tile + 1, buf ^ 1);
            if (tile + 2 < tile1) request(place(tile + 2));
        }
        if (tile * kTileTokens <= pos_last) {
            const q8_u4* k = lds + buf * 2048 + lane;
            q8_float4 s[RB][4];
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int b = 0; b < 4; ++b) s[r][b] = q8_float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const q8_half8 w = __builtin_bit_cast(q8_half8, k[64 * (4 * b + e)]);
#pragma unroll
                    for (int r = 0; r < RB; ++r) s[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, q[r][e], s[r][b], 0, 0, 0);
                }
            // (a factor of zero stands for one so small that every weight is 1: 0 times a masked -infinity is no number)
            const float by = fmaxf(scale * ks, 1e-37f);
            if (tile * kTileTokens + kTileTokens - 1 > pos_first) {
                const int first = tile * kTileTokens + 16 * g;
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[r][i >> 2][i & 3] = first + i > pos[r] ? -INFINITY : s[r][i >> 2][i & 3];
            }
            float top[RB];
            largest_log = fmaxf(largest_log, v_log);
            const float next_log = fmaxf(v_log, largest_log + kFaintest);
            const bool move = v_log > unit_log || (v_log > kNoScale && next_log < unit_log + kFaint);
            bool over = move;
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                float x = s[r][0][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) x = fmaxf(x, s[r][i >> 2][i & 3]);
                top[r] = x * by;
                over |= top[r] > ref[r] + kQ8Slack;
            }
            if (__any(over)) {
                const float v_keep = move ? __builtin_amdgcn_exp2f(unit_log - next_log) : 1.f;
                unit_log = move ? next_log : unit_log;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    top[r] = fmaxf(top[r], __shfl_xor(top[r], 16));
                    top[r] = fmaxf(top[r], __shfl_xor(top[r], 32));
                    const float now = top[r] > ref[r] + kQ8Slack ? top[r] : ref[r], keep = __builtin_amdgcn_exp2f(ref[r] - now);
                    ref[r] = now;
                    sum[r] *= keep;
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[r][c] *= keep * v_keep;
                }
            }
            const float bias = fmaxf(v_log - unit_log, kFaintest), back = __builtin_amdgcn_exp2f(-bias);
            bool wide = false;
#pragma unroll
            for (int r = 0; r < RB; ++r) wide |= fabsf(ref[r]) > 0x1p20f;
            q8_half8 p[RB][2];
            if (__any(wide)) {
                // scores beyond 2^20: as rounded products, in their maximum and here (a fused multiply-add's would differ)
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
#pragma clang fp contract(off)
                        const float x = s[r][i >> 2][i & 3] * by;
                        s[r][i >> 2][i & 3] = (x - ref[r]) + (kQ8Above + bias);
                    }
            } else {
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const float below = kQ8Above + bias - ref[r];
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[r][i >> 2][i & 3] = fmaf(s[r][i >> 2][i & 3], by, below);
                }
            }
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = __builtin_amdgcn_exp2f(s[r][i >> 2][i & 3]);
                    part += w;
                    p[r][i >> 3][i & 7] = (_Float16)w;
                }
                sum[r] = fmaf(part, back, sum[r]);
            }
            const q8_u4* v = lds + buf * 2048 + 1024 + lane;
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const q8_half8 w = __builtin_bit_cast(q8_half8, v[64 * (2 * c + e)]);
#pragma unroll
                    for (int r = 0; r < RB; ++r) o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, p[r][e], o[r][c], 0, 0, 0);
                }
        }
        __syncthreads();
    }

    // ---- lane (col, g) holds channels 16 c + 4 g + e of row col, in units of 2^unit_log
    const float v_unit = __builtin_amdgcn_exp2f(unit_log);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        sum[r] += __shfl_xor(sum[r], 16);
        sum[r] += __shfl_xor(sum[r], 32);
        const int row = row0 + 16 * r + col;
        if (row >= rows) continue;
        const int j = row / qper;
        const size_t to = ((size_t)n * a.m + j) * a.n_q_heads + h * qper + (row - j * qper);
        if (pieces == 1) {
            const float by = sum[r] > 0.f ? v_unit / sum[r] : 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                typedef _Float16 half4 __attribute__((ext_vector_type(4)));
                half4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (_Float16)(o[r][c][e] * by);
                *reinterpret_cast<half4*>(a.out + to * kQ8Head + 16 * c + 4 * g) = y;
            }
        } else {
            float* dst = a.partials + (to * a.n_split + split) * kQ8Partial;
            if (g == 0) {
                dst[0] = ref[r];
                dst[1] = sum[r];
            }
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) dst[kPartialHeader + 16 * c + 4 * g + e] = o[r][c][e] * v_unit;
        }
    }
}

template <int KIND, int WAVES>
cq_status launch(const Q8AttentionArgs& a, hipStream_t stream)
{
    constexpr int ROWS = 16 * RB * WAVES;
    constexpr unsigned smem = 2 * 2 * 16 * 64 * 16;
    static LdsKernelSetup setup;
    if (setup.ensure(reinterpret_cast<const void*>(chunk_q8_kernel<KIND, WAVES>)) != hipSuccess) return CQ_ERR_HIP;
    const int rows = a.m * (a.n_q_heads / a.n_kv_heads), row_blocks = (rows - 1) / ROWS + 1;
    const int64_t units = (int64_t)a.batch * a.n_kv_heads * a.n_split, grid = (units + 7) / 8 * 8 * row_blocks;
    if (grid > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    hipLaunchKernelGGL((chunk_q8_kernel<KIND, WAVES>), dim3((unsigned)grid), dim3(WAVES * 64), smem, stream, a, row_blocks, (unsigned)units);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace

cq_status launch_chunk_q8(const Q8AttentionArgs& a, int kind, int row_block, hipStream_t stream)
{
    if (row_block == 256) return kind == CQ_Q8_INT8 ? launch<CQ_Q8_INT8, 8>(a, stream) : launch<CQ_Q8_E4M3, 8>(a, stream);
    return kind == CQ_Q8_INT8 ? launch<CQ_Q8_INT8, 4>(a, stream) : launch<CQ_Q8_E4M3, 4>(a, stream);
}

}  // namespace cq
