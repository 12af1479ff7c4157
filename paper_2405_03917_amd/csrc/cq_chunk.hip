// Causal attention of the last m tokens of each sequence over its packed CQ cache (a prefill
// chunk, or the verification step of speculative decoding), for gfx950.  Eq. 1 of the paper once
// per query token; the cache already holds the codes of the m tokens.
//
// With many queries per (sequence, KV head) the per-query lookup tables of the decode kernel
// no longer fit on chip and the path becomes a dense contraction, so this one is built on the
// matrix cores: a workgroup (8 wavefronts) owns up to 256 query rows of one KV head (query
// tokens x the query heads that share the KV head), walks the context in 64-token tiles, turns
// each tile's codes back into fp16 keys and values ONCE in LDS (centroid gathers from the
// L2-resident codebooks), and every wavefront runs a flash-attention step on its 32 rows:
//     S^T = K Q^T      v_mfma_f32_32x32x16_f16, A = keys of 32 tokens (LDS), B = queries (registers)
//     online softmax   each lane owns ONE query (a column of S^T): running maximum, sum and the
//                      rescaling of its output column are lane-local
//     O^T += V^T P^T   A = values (LDS, transposed by the read), B = the probabilities just computed,
//                      scaled by 2^12 and split into two fp16 numbers (high and low part: 22
//                      bits; one fp16 alone leaves errors of 1e-5 of the largest output element,
//                      too much for the small ones); fp32 accumulation
// HBM traffic is the codes, read once per workgroup.  Three things take about the same time: the
// matrix cores (rotated keys: 128 products per SIMD and 64-token tile, 4224 clocks), the LDS reads that
// feed them (4600 clocks per CU) and the vector ALU (4900 clocks per SIMD); a tile takes 7500, as two wavefronts
// per SIMD overlap them only in part.  Measured (CQ-8c8b, 32 / 8 heads, 500 rotated query tokens of 2
// sequences x 9001): 384 -> 333 us; 4 x 512 query tokens at 8192, 32 heads: 741 -> 617 us rotated,
// 530 -> 490 us not.  What gave it: straight instruction streams in which products and vector work
// alternate, operands read a group ahead, the queries' loads waited for before the loop, gathers and
// rotation a tile ahead of their use, values kept token by token and transposed by the read, and
// wavefronts that lag before those that lead.  Long contexts with few rows are split over workgroups and
// merged by the decode path's merge kernel (same (m, l, o) partials).
#include <type_traits>

#include "cq_lds_gather.hpp"

namespace cq {
namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));

// 8 wavefronts x 32 query rows per workgroup (one workgroup per CU), or 4 x 32 where a KV head has
// no more than 128 rows (two workgroups per CU then)
constexpr int kKsStride = 272;                    // bytes per token row of the key tile (256 + 16: conflict-free 16-byte reads)
constexpr int kKsBytes = kTileTokens * kKsStride; // 17408
// The value tile has a token's 128 channels in a row too, its four 64-byte quarters exchanged by the token's two
// low bits: the transposing read takes a quarter of four tokens at a time, which then lie in different banks.
constexpr int kVsStride = 256;
constexpr int kVsBytes = kTileTokens * kVsStride; // 16384
// a stage: the key tile, the value tile and (rotated keys only) the low parts of the key tile
constexpr int kStageBytes(bool rope) { return kKsBytes + kVsBytes + (rope ? kKsBytes : 0); }
constexpr unsigned kRawBase(bool rope) { return 2 * kStageBytes(rope); }     // behind the two stages: the raw code tiles (K, V) of two tiles
constexpr unsigned kAngleBytes = 64 * kTileTokens * 8;                       // behind those (rotated keys): cos / sin per pair and token of a tile
typedef __attribute__((address_space(3))) u32x4 lds_q;

__device__ __forceinline__ half8_t lds_half8(unsigned byte_addr)
{
    return *(__attribute__((address_space(3))) half8_t*)(byte_addr);
}
// two numbers as fp16 plus what fp16 leaves of them
__device__ __forceinline__ void split_pair(float x, float y, unsigned& high, unsigned& low)
{
    const half2_t h = __builtin_convertvector(float2_t{x, y}, half2_t);
    float minus = -1.f;                 // (opaque: as a product the difference is one instruction with its conversions)
    asm("" : "+s"(minus));
    half2_t l;
    l.x = (_Float16)__builtin_fmaf((float)h.x, minus, x);
    l.y = (_Float16)__builtin_fmaf((float)h.y, minus, y);
    high = __builtin_bit_cast(unsigned, h);
    low = __builtin_bit_cast(unsigned, l);
}
// the larger of lane i's and lane (i ^ 32)'s value
__device__ __forceinline__ float half_wave_max(float x)
{
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Codes of 64 tokens -> fp16 keys and values [token][channel] in LDS.
// The codes of a tile first go to LDS as they are (request_codes / store_codes: one 16-byte record per
// thread).  Then thread (token u = tid % 64, wavefront e = tid / 64) expands groups
// e Gh/NW .. (e + 1) Gh/NW - 1 of its token: the code of group g sits in slot (g - u) mod Gh of the
// token's record.  A wavefront thus gathers from ONE group's centroids at a time: its 64 lanes
// touch the 8 to 32 cache lines of that group's table instead of 64 lines of 64 tables, which is
// what the texture path charges for.  Neighbouring groups of one thread also make its stores 16
// bytes wide for every format.
//
// ROPE (keys cached before the rotary position embedding): thread (u, e) takes half as many
// neighbouring groups from each half of the head instead, so that it holds both halves of its channel
// pairs (channel i of the head is rotated with channel i + 64, i.e. group g with group g + Gh/2), and
// rotate() turns the pairs to the token's position before the keys go to LDS: once per (tile, KV
// head), for all query rows of the workgroup.
template <int GH, int C, int NW, int B, bool ROPE>
struct Dequant {
    static constexpr int GPT = GH / NW;                 // groups per thread
    static_assert(!ROPE || GPT % 2 == 0, "a thread holds both groups of a pair");
    static constexpr int NP = ROPE ? GPT / 2 * C : 1;   // channel pairs per thread
    float2 ts[NP];                                      // ROPE: cos / sin of (first position of the tile * theta) of this thread's pairs
    // ROPE: low parts of the rotated keys.  A rotated key is kept as the sum of two fp16 numbers
    // (22 bits): rounded to one, its error of 2^-11 reaches the scores and leaves 4e-4 of a
    // row's largest output element, which fails the 2e-3 bar on the small elements
    unsigned kwl[GPT][C / 2];
    __device__ __forceinline__ static int group(int e, int gi)
    {
        return ROPE ? (gi < GPT / 2 ? 0 : GH / 2) + e * (GPT / 2) + gi % (GPT / 2) : e * GPT + gi;
    }
    static constexpr int K = 1 << B;                    // centroids per group
    static constexpr int TILE = kTileTokens * GH * B / 8;   // bytes of one tile's codes (b = 10: low bytes, then high-bit words)
    static constexpr int LOADERS = TILE / 16;           // threads that carry one record of K and one of V
    static constexpr int RAW_STAGE = 2 * TILE;          // K tile, V tile
    static_assert(LOADERS <= NW * 64, "one record per thread");
    struct Codes {
        u32x4 k, v;
    };
    Codes raw;                                          // 16-byte records of codes on their way to LDS
    unsigned kw[GPT][C / 2], vw[GPT][C / 2];            // the centroids of this thread's (token, group) pairs

    __device__ __forceinline__ static Codes request_codes(const uint8_t* ktile, const uint8_t* vtile, int tid)
    {
        Codes c = {};
        if (tid < LOADERS) {
            c.k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(ktile) + tid);
            c.v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vtile) + tid);
        }
        return c;
    }
    __device__ __forceinline__ static void store_codes(const Codes& c, unsigned k_slot, unsigned v_slot, int tid)
    {
        if (tid < LOADERS) {
            *(lds_q*)(k_slot + (unsigned)tid * 16) = c.k;
            *(lds_q*)(v_slot + (unsigned)tid * 16) = c.v;
        }
    }

    // this thread's codes from the raw tile, and the request for their centroids (L2-resident codebooks)
    unsigned code[GPT];
    __device__ __forceinline__ void read_codes(unsigned raw, int tid)
    {
        typedef __attribute__((address_space(3))) uint8_t lds_b;
        const int u = tid & 63, e = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
        for (int gi = 0; gi < GPT; ++gi) {
            const unsigned slot = (unsigned)(group(e, gi) - u) & (unsigned)(GH - 1);
            code[gi] = *(lds_b*)(raw + (slot >> 4) * 1024 + (unsigned)u * 16 + (slot & 15));
            if constexpr (B == 10) {        // bits [2 s + 1 : 2 s] of the token's high-bit word
                typedef __attribute__((address_space(3))) unsigned lds_w;
                code[gi] |= ((*(lds_w*)(raw + (unsigned)(kTileTokens * GH) + (unsigned)u * 4) >> (2 * slot)) & 3u) << 8;
            }
        }
    }
    // (not `wanted`: zeros, not the old contents, which would occupy their registers until here)
    __device__ __forceinline__ void request(unsigned (&w)[GPT][C / 2], const uint16_t* c_head, int tid, bool wanted) const
    {
        const int e = __builtin_amdgcn_readfirstlane(tid >> 6);
        if (wanted) {
#pragma unroll
            for (int gi = 0; gi < GPT; ++gi) {
                const unsigned* src = reinterpret_cast<const unsigned*>(c_head + ((size_t)group(e, gi) * K + code[gi]) * C);
#pragma unroll
                for (int i = 0; i < C / 2; ++i) w[gi][i] = src[i];
            }
        } else {
#pragma unroll
            for (int gi = 0; gi < GPT; ++gi)
#pragma unroll
                for (int i = 0; i < C / 2; ++i) w[gi][i] = 0;
        }
    }
    __device__ __forceinline__ void gather(unsigned (&w)[GPT][C / 2], unsigned raw, const uint16_t* c_head, int tid, bool wanted)
    {
        read_codes(raw, tid);
        request(w, c_head, tid, wanted);
    }

    // ROPE: the angle of a rotation is the sum of two: u theta_i per lane, whose cos / sin lie in LDS ([pair][lane]),
    // and 64 tile theta_i, the same for the wavefront (read in the constant address space, i.e. through the scalar
    // cache: the table is older than this kernel)
    __device__ __forceinline__ void request_tile_angles(const float2* tile_tab, int tile, int tid)
    {
        if constexpr (ROPE) {
            const int e = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                typedef const __attribute__((address_space(4))) float* scalar_floats;
                const scalar_floats t = (scalar_floats)(tile_tab + (size_t)tile * 64 + e * NP + p);
                ts[p] = make_float2(t[0], t[1]);
            }
        }
    }
    struct Angles {
        float2 c0, c1;
    };
    __device__ __forceinline__ static Angles lane_angles(unsigned table, int tid, int q)
    {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) f32x2 lds_f2;
        const unsigned at = table + (unsigned)(__builtin_amdgcn_readfirstlane(tid >> 6) * NP + 2 * q) * 512 + (unsigned)(tid & 63) * 8;
        const f32x2 x = *(lds_f2*)at, y = *(lds_f2*)(at + 512);
        return {make_float2(x.x, x.y), make_float2(y.x, y.y)};
    }
    // the same from the table in memory
    __device__ __forceinline__ static Angles table_angles(const float2* lane_tab, int tid, int q)
    {
        const float2* t = lane_tab + (size_t)(__builtin_amdgcn_readfirstlane(tid >> 6) * NP + 2 * q) * 64 + (tid & 63);
        return {t[0], t[64]};
    }
    // rotate pairs 2 q and 2 q + 1 of the gathered keys:
    // (k_i, k_{i+64}) -> (k_i cos - k_{i+64} sin, k_{i+64} cos + k_i sin), fp32, then two fp16 parts
    __device__ __forceinline__ void rotate(const Angles& lane_part, int q)
    {
        if constexpr (ROPE) {
            const int gi = q / (C / 2), i = q % (C / 2);
            auto sum = [](float2 t, float2 l) { return make_float2(t.x * l.x - t.y * l.y, t.y * l.x + t.x * l.y); };
            const float2 c0 = sum(ts[2 * q], lane_part.c0), c1 = sum(ts[2 * q + 1], lane_part.c1);
            const half2_t lo = __builtin_bit_cast(half2_t, kw[gi][i]), hi = __builtin_bit_cast(half2_t, kw[gi + GPT / 2][i]);
            const float fl0 = (float)lo.x * c0.x - (float)hi.x * c0.y, fh0 = (float)hi.x * c0.x + (float)lo.x * c0.y;
            const float fl1 = (float)lo.y * c1.x - (float)hi.y * c1.y, fh1 = (float)hi.y * c1.x + (float)lo.y * c1.y;
            split_pair(fl0, fl1, kw[gi][i], kwl[gi][i]);
            split_pair(fh0, fh1, kw[gi + GPT / 2][i], kwl[gi + GPT / 2][i]);
            // (here, between the products, not behind them)
            asm volatile("" : "+v"(kw[gi][i]), "+v"(kwl[gi][i]), "+v"(kw[gi + GPT / 2][i]), "+v"(kwl[gi + GPT / 2][i]));
        }
    }
    static constexpr int kRotations = ROPE ? GPT / 2 * (C / 2) : 0;

    // the thread's channels in 16-byte pieces (eight channels; its groups lie side by side, in each half of the head
    // for rotated keys), the values first
    static constexpr int PIECES = GPT * C / 8;
    __device__ __forceinline__ static int first_channel(int e, int q)
    {
        return ROPE ? (q < PIECES / 2 ? 0 : 64) + e * (GPT / 2 * C) + 8 * (q % (PIECES / 2)) : e * (GPT * C) + 8 * q;
    }
    __device__ __forceinline__ static u32x4 piece(const unsigned (&w)[GPT][C / 2], int q)
    {
        constexpr int H = C / 2;
        return u32x4{w[(4 * q) / H][(4 * q) % H], w[(4 * q + 1) / H][(4 * q + 1) % H], w[(4 * q + 2) / H][(4 * q + 2) % H],
                     w[(4 * q + 3) / H][(4 * q + 3) % H]};
    }
    __device__ __forceinline__ void store_values(unsigned stage, int tid) const
    {
        const int u = tid & 63, e = __builtin_amdgcn_readfirstlane(tid >> 6);
        const unsigned row = stage + kKsBytes + (unsigned)u * kVsStride;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) *(lds_q*)(row + ((unsigned)(first_channel(e, q) * 2) ^ ((unsigned)(u & 3) << 6))) = piece(vw, q);
    }
    __device__ __forceinline__ void store_keys(unsigned stage, int tid) const
    {
        const int u = tid & 63, e = __builtin_amdgcn_readfirstlane(tid >> 6);
        const unsigned row = stage + (unsigned)u * kKsStride;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            *(lds_q*)(row + (unsigned)(first_channel(e, q) * 2)) = piece(kw, q);
            if constexpr (ROPE) *(lds_q*)(row + (unsigned)(kKsBytes + kVsBytes + first_channel(e, q) * 2)) = piece(kwl, q);
        }
    }
};

// 8 wavefronts are two per SIMD; of the workgroups of 4, two fit on a CU by their LDS but for rotated keys and
// the code tiles of CQ-2c8b: those take the registers of two wavefronts
constexpr int chunk_waves_per_simd(int c, int nw, bool rope) { return nw == 4 && (rope || c == 2) ? 1 : 2; }

// SHORT: pieces of the context of up to kShortTiles tiles, without the look-ahead of the pipeline, whose registers
// (the form of four wavefronts spills some) and prologue such a call does not repay.  Not rotated, pipeline / this:
// CQ-8c8b 64 x 64 tokens over 64: 39.6 / 35.3 us, 40 x 70 over 100: 36.4 / 32.1, 16 x 100 over 190: 20.2 / 18.7,
// CQ-8c10b 43.4 / 37.5, 41.6 / 36.5 and 24.3 / 24.2; over four tiles the pipeline is ahead.  Rotated keys, whose
// pipeline repays itself from two tiles on: CQ-8c8b 64 x 64 over 64: 66.2 / 64.9.
constexpr int kShortTiles(bool rope) { return rope ? 1 : 3; }

#define CQ_VIEW_KERNEL 0
#include "cq_chunk_kernel.hpp"
#undef CQ_VIEW_KERNEL
#define CQ_VIEW_KERNEL 1
#include "cq_chunk_kernel.hpp"
#undef CQ_VIEW_KERNEL

template <int GH, int C, int NW, int B, bool ROPE, bool SHORT, class Args>
constexpr auto chunk_variant()
{
    if constexpr (std::is_same_v<Args, ChunkArgs>) return chunk_attention_kernel<GH, C, NW, B, ROPE, SHORT>;
    else return chunk_attention_window_kernel<GH, C, NW, B, SHORT>;
}

template <int GH, int C, int NW, int B, bool ROPE, bool SHORT, class Args>
cq_status launch_chunk_variant(const Args& a, hipStream_t stream)
{
    constexpr auto kernel = chunk_variant<GH, C, NW, B, ROPE, SHORT, Args>();
    static LdsKernelSetup setup;
    if (setup.ensure(reinterpret_cast<const void*>(kernel)) != hipSuccess) return CQ_ERR_HIP;
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int row_blocks = (a.m * qper + NW * 32 - 1) / (NW * 32);
    const unsigned grid = (unsigned)(a.batch * a.n_split * row_blocks * a.f.n_kv_heads);
    const size_t lds = 2 * kStageBytes(ROPE) + (SHORT ? kShortTiles(ROPE) : 2) * Dequant<GH, C, NW, B, ROPE>::RAW_STAGE +
                       (ROPE && !SHORT ? kAngleBytes : 0);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(NW * 64), lds, stream, a);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

int walked_tiles(const ChunkArgs& a) { return (a.t + kTileTokens - 1) / kTileTokens; }
int walked_tiles(const ChunkViewArgs& a) { return view_tiles(a.t, a.m, a.window, a.n_sink); }

template <int GH, int C, int NW, int B, bool ROPE, class Args>
cq_status launch_chunk_tiles(const Args& a, hipStream_t stream)
{
    const int n_tiles = walked_tiles(a);
    if ((a.tiles_per_split < n_tiles ? a.tiles_per_split : n_tiles) <= kShortTiles(ROPE)) return launch_chunk_variant<GH, C, NW, B, ROPE, true>(a, stream);
    return launch_chunk_variant<GH, C, NW, B, ROPE, false>(a, stream);
}

template <int GH, int C, int B, class Args>
cq_status launch_chunk_rows(const Args& a, hipStream_t stream)
{
    const int rows = a.m * (a.n_q_heads / a.f.n_kv_heads);
    if constexpr (std::is_same_v<Args, ChunkArgs>) {
        if (a.rope_tile_tab) {
            if (chunk_rows_per_workgroup(rows) == 128) return launch_chunk_tiles<GH, C, 4, B, true>(a, stream);
            return launch_chunk_tiles<GH, C, 8, B, true>(a, stream);
        }
    }
    if (chunk_rows_per_workgroup(rows) == 128) return launch_chunk_tiles<GH, C, 4, B, false>(a, stream);
    return launch_chunk_tiles<GH, C, 8, B, false>(a, stream);
}

template <class Args>
cq_status launch_chunk_format(const Args& a, hipStream_t stream)
{
    cq_status st = CQ_ERR_UNSUPPORTED;
    if (a.f.b == 8 && a.f.head_dim == 128) {
        if (a.f.gh == 16 && a.f.c == 8) st = launch_chunk_rows<16, 8, 8>(a, stream);
        else if (a.f.gh == 32 && a.f.c == 4) st = launch_chunk_rows<32, 4, 8>(a, stream);
        else if (a.f.gh == 64 && a.f.c == 2) st = launch_chunk_rows<64, 2, 8>(a, stream);
    } else if (a.f.b == 10 && a.f.head_dim == 128 && a.f.gh == 16 && a.f.c == 8) {
        st = launch_chunk_rows<16, 8, 10>(a, stream);
    }
    if (st != CQ_OK) return st;
    if (a.n_split > 1)
        return launch_decode_merge(a.partials, a.out, a.batch * a.m * a.n_q_heads, a.n_q_heads, (int64_t)a.n_q_heads * a.f.head_dim, a.n_split,
                                   a.f.head_dim, stream);
    return CQ_OK;
}

}  // namespace

int chunk_rows_per_workgroup(int rows_per_kv_head) { return rows_per_kv_head <= 128 ? 128 : 256; }

cq_status launch_chunk_attention(const ChunkArgs& a, hipStream_t stream) { return launch_chunk_format(a, stream); }
cq_status launch_chunk_attention_window(const ChunkViewArgs& a, hipStream_t stream) { return launch_chunk_format(a, stream); }

}  // namespace cq
