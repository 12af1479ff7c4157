// Attention over the 8-bit block cache (cq_decode_attention_q8, cq_chunk_attention_q8) for few rows per KV head, and the merge of
// context pieces, for gfx950.
//
//   s = scale k_scale (q . k_code),  p = 2^(s log2(e) - ref),  out = sum_tiles v_scale sum_i p_i v_code_i / sum_i p_i
//
// A wavefront walks whole tiles by itself, everything in registers: S^T = K Q^T and O^T = V^T P^T by 16x16x32 products, rows of the
// KV head (query heads of a token, tokens of a chunk) in the 16 columns.  The result of S^T holds, in the lane of column n
// and block g, rows 4 g + e; rows of key tile b are tokens 16 g + 4 b + e, so a lane's scores of b = 0 .. 3 are tokens 16 g .. 16 g + 15, in
// order: what the lane feeds into the second product, whose other operand (16 tokens of a channel) is 16 bytes of the cache as they lie.
// Bound by memory: 16 KB a tile against 512 products' clocks and about 1000 of conversions.  16 x 32 streams of 8192 tokens, 1.07 GB: 178 us,
// 6.0 TB/s of the 6.4 that a large read reaches; 24 x 8 of 6007 at most, paged e4m3, 167 MB: 43 us, 3.9; 8 of 2000, 4 MB: 9.0 us, most of it the
// way of a first request and of the merge.
#include <algorithm>

#include "cq_q8.hpp"

namespace cq {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
// Partial rows go from workgroup to workgroup two floats at a time; within a running kernel by device-scope accesses, written through
// to where every workgroup's loads find them.
typedef float float2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put2(float* p, float x, float y, bool within)
{
    if (!within) *reinterpret_cast<float2_t*>(p) = float2_t{x, y};
    else __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, float2_t{x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <bool WITHIN>
__device__ __forceinline__ float2_t get2(const float* p)
{
    if (!WITHIN) return *reinterpret_cast<const float2_t*>(p);
    return __builtin_bit_cast(float2_t, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Rows row0 .. row0 + count - 1 (32 at most) of a stream from their `pieces` partials (reference, sum, 128 channels), by a workgroup: 16
// lanes take 8 channels each of a row, or, of few rows, of every second, fourth, ... of its pieces.  One pass with a running
// reference, requests of four pieces together; then those of a row meet in LDS, and are rounded to fp16 once.
struct MergeLds {
    float part[16][16][10];                                 // [group][lane]: reference, sum, channels
};
template <bool WITHIN>
__device__ __forceinline__ void merge_rows(const Q8AttentionArgs& a, int n, int h, int row0, int count, int pieces, MergeLds& lds, int tid)
{
    const int qper = a.n_q_heads / a.n_kv_heads, group = tid >> 4, lane = tid & 15;
    const int share = count <= 1 ? 16 : count <= 2 ? 8 : count <= 4 ? 4 : count <= 8 ? 2 : 1;
    const int first = group / share, at_once = 16 / share;  // rows first, first + at_once, ...
    for (int base = 0; base < count; base += at_once) {
        const int row = row0 + base + first, j = row / qper;
        const bool mine = base + first < count;
        const size_t at = ((size_t)n * a.m + j) * a.n_q_heads + h * qper + (row - j * qper);
        float m = kQ8Lowest, l = 0.f, y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
        if (mine) {
            const float* p = a.partials + (at * a.n_split + group % share) * kQ8Partial;
#pragma unroll 4
            for (int s = group % share; s < pieces; s += share, p += share * kQ8Partial) {
                const float2_t head = get2<WITHIN>(p);
                float2_t x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = get2<WITHIN>(p + kPartialHeader + 8 * lane + 2 * e);
                const float now = fmaxf(m, head[0]), keep = __builtin_amdgcn_exp2f(m - now), w = __builtin_amdgcn_exp2f(head[0] - now);
                l = fmaf(l, keep, head[1] * w);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(y[e], keep, x[e >> 1][e & 1] * w);
                m = now;
            }
        }
        if (share > 1) {
            __syncthreads();
            float* mine_at = lds.part[group][lane];
            mine_at[0] = m;
            mine_at[1] = l;
#pragma unroll
            for (int e = 0; e < 8; ++e) mine_at[2 + e] = y[e];
            __syncthreads();
            if (group % share == 0) {
                for (int s = 1; s < share; ++s) {
                    const float* x = lds.part[group + s][lane];
                    const float now = fmaxf(m, x[0]), keep = __builtin_amdgcn_exp2f(m - now), w = __builtin_amdgcn_exp2f(x[0] - now);
                    l = fmaf(l, keep, x[1] * w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = fmaf(y[e], keep, x[2 + e] * w);
                    m = now;
                }
            }
        }
        if (mine && group % share == 0) {
            q8_half8 z;
            const float by = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (_Float16)(y[e] * by);
            *reinterpret_cast<q8_half8*>(a.out + at * kQ8Head + 8 * lane) = z;
        }
    }
}

// A workgroup per 32 rows (16, where a workgroup of the kernel in front served as many).
__global__ __launch_bounds__(kThreads) void merge_q8_kernel(Q8AttentionArgs a, int blocks, int block_rows)
{
    __shared__ MergeLds lds;
    const int block = blockIdx.x % blocks, stream = blockIdx.x / blocks;
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads, row0 = block * block_rows;
    const int pieces = a.pieces(a.block_tiles(a.length(n), row0 / a.row_block));
    if (pieces > 1) merge_rows<false>(a, n, h, row0, min(block_rows, a.m * (a.n_q_heads / a.n_kv_heads) - row0), pieces, lds, threadIdx.x);
}

template <int KIND, int RB>
__global__ __launch_bounds__(kThreads, 2) void rows_q8_kernel(Q8AttentionArgs a, int row_blocks, unsigned units)
{
    __shared__ float lds[kWaves][16 * RB][kQ8Partial];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    // the row blocks of a piece of a stream run on one XCD, which shares what it reads; all streams' first pieces are dealt out, then all
    // second ones: the heads of a sequence have the same pieces to do, and the XCDs as many of them each
    const unsigned eighth = blockIdx.x >> 3;
    const int block = eighth % row_blocks;
    const unsigned unit = (eighth / row_blocks) * 8 + (blockIdx.x & 7);
    if (unit >= units) return;
    const unsigned streams = (unsigned)(a.batch * a.n_kv_heads);
    const int split = unit / streams, stream = unit % streams;
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads;
    const int qper = a.n_q_heads / a.n_kv_heads, rows = a.m * qper, row0 = block * 16 * RB;
    const int t_n = a.length(n), pos0 = t_n - a.m, pos_first = pos0 + row0 / qper;
    const int n_tiles = a.block_tiles(t_n, block), pieces = a.pieces(n_tiles);
    if (split >= pieces) return;
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

    // Codes of a tile: the next one's keys and values each take the place of those they follow.  (Two tiles' registers, all of the next
    // requested ahead of this one's work, are 2 wavefronts a SIMD instead of 3: 8 streams of 2000 tokens 9.1 -> 8.4 us, of 65536 27.6 -> 28.6, 64 of 32768,
    // e4m3, 95.4 -> 98.6, 32 of 4096 12.3 -> 13.1.)
    q8_u4 kr[8], vr[8];
    auto request_keys = [&](size_t at) {
        const uint8_t* src = a.cache.codes[0] + at * kQ8TileBytes + (16 * (col >> 2) + (col & 3)) * kQ8Head + 16 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) kr[i] = *reinterpret_cast<const q8_u4*>(src + 4 * (i >> 1) * kQ8Head + 64 * (i & 1));
    };
    auto request_values = [&](size_t at) {
        const uint8_t* src = a.cache.codes[1] + at * kQ8TileBytes + col * kTileTokens + 16 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) vr[i] = *reinterpret_cast<const q8_u4*>(src + 16 * i * kTileTokens);
    };
    // lane i knows where the i-th of this wavefront's tiles (64 at most: kQ8RowTiles) lies, and its scales: none is asked for by itself
    // (those behind the sequence's end lie somewhere in the pool, unused; its length is not waited for)
    const int count = max(tile1 - tile0 - wave + kWaves - 1, 0) / kWaves;
    const size_t places = a.cache.map.tile_index(n, h, min(tile0 + wave + kWaves * lane, (a.t - 1) / kTileTokens));
    const float k_scales = a.cache.scales[0][places], v_scales = a.cache.scales[1][places];
    auto place = [&](int i) {
        return (size_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)places, i) | (size_t)(unsigned)__builtin_amdgcn_readlane((int)(places >> 32), i) << 32;
    };
    auto scale_of = [&](float scales, int i) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scales), i)); };
    if (count > 0) {
        request_keys(place(0));
        request_values(place(0));
    }
#pragma unroll 1
    for (int t = 0; t < count; ++t) {
        const int tile = tile0 + wave + kWaves * t;
        const bool more = t + 1 < count;
        const size_t next = place(more ? t + 1 : t);
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
        const float by = fmaxf(scale * scale_of(k_scales, t), 1e-37f);
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
        const float vs = scale_of(v_scales, t);
        // e4m3 bytes of tokens that are not there may be no numbers, and a weight of zero would not hide them
        q8_u4 there = {~0u, ~0u, ~0u, ~0u};
        if (KIND == CQ_Q8_E4M3 && (tile + 1) * kTileTokens > t_n) there = q8_only_before(there, t_n - first);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const q8_u4 w = KIND == CQ_Q8_E4M3 ? vr[c] & there : vr[c];
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
        if (pieces == 1) {
            q8_half8 z;
            const float by = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = (_Float16)(y[i] * by);
            *reinterpret_cast<q8_half8*>(a.out + at * kQ8Head + i0) = z;
        } else {
            float* dst = a.partials + (at * a.n_split + split) * kQ8Partial;
            if ((tid & 15) == 0) put2(dst, m, l, a.counters);
#pragma unroll
            for (int i = 0; i < 8; i += 2) put2(dst + kPartialHeader + i0 + i, y[i], y[i + 1], a.counters);
        }
    }
    if (pieces == 1 || !a.counters) return;
    // ---- the last piece to finish merges them all: every wavefront waits for its stores (a barrier does not), all meet, one
    // thread counts the workgroup in, and the last of them takes the counter back to zero for the next call
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    unsigned* flag = reinterpret_cast<unsigned*>(&lds[0][0][0]);
    if (tid == 0) {
        unsigned* counter = a.counters + (size_t)stream * row_blocks + block;
        const bool last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)pieces - 1u;
        if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = last;
    }
    __syncthreads();
    if (*flag == 0u) return;
    static_assert(sizeof(MergeLds) <= sizeof(lds), "the merge takes the rows' place");
    __syncthreads();                                        // (the flag is read)
    merge_rows<true>(a, n, h, row0, min(16 * RB, rows - row0), pieces, *reinterpret_cast<MergeLds*>(&lds[0][0][0]), tid);
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
    // Up to 64 rows of a KV head go by themselves, 16 to a workgroup where the contexts are few tiles (more of them run, and the
    // codes, read twice, come out of L2), 32 where they are many; more rows share converted tiles through LDS (cq_q8_chunk.hip), where they
    // are enough work for that.  16 | 32 to a workgroup, us: integers, 32 heads, 20 rows of 4096 16.3 | 20.1, 8 heads, 2 x 64 of 4096 16.9 | 21.4;
    // 16 x 32 heads, 20 of 4096 117 | 94, 64 x 32, 17 of 300 53 | 47.  32 | 128: 4 x 32 heads, 128 of 2048 31.8 | 41.4, 8 heads, 512 of 4096 26.3 | 27.9,
    // 8 x 8, 200 of 2000 31 | 35; 8 heads, 512 of 30000 98 | 84, 32 heads, 128 of 16384 65 | 61.
    // Workgroups of eight wavefronts convert a tile half as often as those of four, and reach further in front of their first row and
    // behind their last: where most of the context lies in front of the chunk.  128 -> 256 rows, us: integers, 32 heads, 512 of 16384
    // 163 -> 155, e4m3, 2 x 1024 of 8192 292 -> 272, 32 / 8 heads, 4 x 512 of 16384 558 -> 523; integers, 32 heads, 2 x 4096 of 4096 309 -> 308, 2000 of
    // 2000 60 -> 72, ragged 8 x 1024 of 3000 246 -> 256.
    const int64_t context = (int64_t)batch * n_kv_heads * n_tiles;
    if (rows <= 64) p.row_block = rows <= 16 || context <= 4096 ? 16 : 32;
    else if (rows <= 512 && rows * context <= 1 << 19) p.row_block = 32;
    else p.row_block = rows >= 512 && t - m >= 4096 ? 256 : 128;
    if (tokens_per_split) {
        p.tiles_per_split = p.row_block > 32 ? tokens_per_split / kTileTokens : std::min(tokens_per_split / kTileTokens, kQ8RowTiles);
    } else if (p.row_block > 32) {
        const int64_t blocks = (int64_t)batch * n_kv_heads * ((rows + p.row_block - 1) / p.row_block);
        const int64_t pieces = std::max<int64_t>(1, std::min<int64_t>((n_tiles + 7) / 8, 65536 / p.row_block / blocks));
        p.tiles_per_split = (int)((n_tiles + pieces - 1) / pieces);
    } else {
        // A workgroup costs about 5 us besides its tiles (its way to the first codes, its partials), so there is one round of them: two to
        // a CU, or one where there are few streams, whose pieces then are fewer to merge.  us by workgroups: 24 x 8 streams of 6007 at
        // most, e4m3, 192 53, 384 45, 576 43, 1152 43, 2304 44; 8 of 65536 128 39, 256 28, 512 28, 1024 31, 2048 38; 32 of 4096 128 14, 256 12,
        // 512 13; 512 of 8192 512 178, 1024 185, 4096 188.
        const int64_t blocks = (int64_t)batch * n_kv_heads * ((rows + p.row_block - 1) / p.row_block);
        const int64_t wanted = blocks >= 64 ? (512 + blocks / 2) / blocks : (255 + blocks) / blocks;
        const int64_t pieces = std::max<int64_t>(1, std::min<int64_t>((n_tiles + kWaves - 1) / kWaves, wanted));
        const int64_t tiles = (n_tiles + pieces - 1) / pieces;
        p.tiles_per_split = (int)std::min<int64_t>((tiles + kWaves - 1) / kWaves * kWaves, kQ8RowTiles);
    }
    p.n_split = (n_tiles - 1) / p.tiles_per_split + 1;
    return p;
}

cq_status launch_attention_q8(const Q8AttentionArgs& args, int kind, const Q8Plan& plan, hipStream_t stream)
{
    Q8AttentionArgs a = args;
    a.row_block = plan.row_block;
    const bool chunk = plan.row_block > 32;
    const int64_t blocks = (int64_t)a.batch * a.n_kv_heads * ((a.m * (a.n_q_heads / a.n_kv_heads) - 1) / plan.row_block + 1);
    // Merging within the kernel saves a launch, and costs the way of the partials to memory and back, by a single workgroup: where they are
    // few.  us, apart -> within: 1 row of 128 streams, 4 pieces 24.7 -> 22.8, 4 rows of 8, 8 pieces 9.6 -> 9.1, of 192, 3 pieces 45.9 -> 44.7; 16 rows of
    // 128, 4 pieces 32.3 -> 33.3, 32 of 32, 8 pieces 34.9 -> 39.2; 4 rows of 8 streams, 32 pieces 10.4 -> 12.
    const int block_rows = std::min(a.m * (a.n_q_heads / a.n_kv_heads), std::min(plan.row_block, 32));
    a.counters = chunk || a.n_split == 1 || a.n_split > 8 || block_rows * a.n_split > 32 || blocks > 0x7fffffff ? nullptr : merge_counters_for(stream, (int)blocks);
    const cq_status st = chunk                 ? launch_chunk_q8(a, kind, plan.row_block, stream)
                         : kind == CQ_Q8_INT8 ? launch_rows<CQ_Q8_INT8>(a, plan.row_block, stream) : launch_rows<CQ_Q8_E4M3>(a, plan.row_block, stream);
    if (st != CQ_OK || a.n_split == 1 || a.counters) return st;
    const int per_merge = std::min(plan.row_block, 32), row_blocks = (a.m * (a.n_q_heads / a.n_kv_heads) - 1) / per_merge + 1;
    const int64_t grid = (int64_t)a.batch * a.n_kv_heads * row_blocks;
    if (grid > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    hipLaunchKernelGGL(merge_q8_kernel, dim3((unsigned)grid), dim3(kThreads), 0, stream, a, row_blocks, per_merge);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace cq
