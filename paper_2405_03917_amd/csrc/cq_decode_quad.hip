// Decode attention with grouped queries, both codebooks of a KV head in LDS, for gfx950: the (up to) four query heads
// of a KV head that a workgroup serves share every code load, every gathered key and value and (keys cached before the
// rotary embedding) every key rotation.  The formats whose two codebooks fit: CQ-8c8b and CQ-4c8b (2 x 64 KB of the
// CU's 160 KB).
//
// A codebook belongs to the KV head and not to the sequence, so a workgroup brings both in ONCE and then walks
// (sequence, split) items of its KV head; no table is built per sequence and query head.  Within an item every
// wavefront takes every eighth 64-token tile by itself, keys, softmax and values, with no barrier in the loop:
//   scores   lane = token.  A lane reads the centroids of its token's codes (ds_read_b128 / b64); a product of four
//            heads x 4 channels with 4 channels x 4 tokens per block of four lanes (v_mfma_f32_4x4x4_16B_f16, the
//            queries broadcast from one block) leaves a token's four scores in its lane's four registers.
//            ROPE: the key is rotated by the lane's part of its position and each head's query by the tile's
//            (cq_decode_rope.hip), products of one channel each in fp32 (v_mfma_f32_4x4x1_16B_f32).
//   softmax  relative to a running reference per head that moves only when a score exceeds it by 3 (factor 8):
//            probabilities scaled by 2^12, three fp16 parts each (33 bits), twelve of sixteen columns of a
//            [token][column] array in LDS, read back transposed
//   values   O^T[channel][column] += V^T[channel][token] P[token][column], v_mfma_f32_16x16x32_f16; the transposing
//            read gathers the centroids of 4 tokens per lane group
// The wavefronts are merged through LDS at the end of an item; the partials of several splits by a kernel of its own
// (counting workgroups in and merging in the last of them, as cq_decode.hip does, took 1 to 3 us longer here).
//
// Bound, keys as stored: the LDS.  A tile costs a CU 434 (CQ-8c8b) or 476 (CQ-4c8b) clocks of it, 270 to 320 of them bank
// conflicts of the gathers: 64 random 8-byte entries take 6.2 to 7 clocks instead of 2, 16-byte ones 12 instead of 4 (other
// places of the entries, by group or code, 5.7 to 6.4).  Measured: the paged fused step of CQ-4c8b, 32 / 8 heads, 24 ragged
// rows to 6007, 44.4 us with a workgroup and tables per query head -> 30.5 here: launch 2.7, codebooks 2.8, search for the
// new token's codes 3, 22 for the 94 tiles of the longest row (LDS busy throughout), merge 1.
// ROPE: issue of vector and matrix instructions, 576 and 144 per tile, which hardly overlap: 2304 + 1280 of 3800 clocks per
// tile and SIMD.  The fused step of CQ-8c8b, 32 / 8 heads, 32 x 16384: 161.4 us with the phases one after the other in a
// workgroup (scores of a split to LDS, the value codebook in the key codebook's place) -> 112.  On the way: splits
// that one workgroup walks joined 143 -> 121; priorities 121 -> 116; nothing spilled ahead of the first requests 118 -> 112.
// Priorities: the two wavefronts of a SIMD should be in different phases, and neither may fall behind (an item ends
// with its slowest wavefront).  A wavefront's priority is high in its latency-bound half of a tile (softmax, values), and
// within both halves the wavefronts take turns from tile to tile: with none, wavefront 0 waited 26 of 130 us for the
// others of its workgroup; now 2.5.
#include <type_traits>

#include "cq_decode_split.hpp"
#include "cq_key_gather.hpp"
#include "cq_lds_gather.hpp"

namespace cq {
namespace {

constexpr int kQuadThreads = 512;
constexpr int kQuadHeads = 4;
constexpr int kQuadWaves = kQuadThreads / 64;
// LDS: key codebook, value codebook, per wavefront 2 KB (probabilities of a tile, 64 tokens x 16 columns; at the end of
// an item its four output rows), the wavefronts' (reference, sum) pairs, the new token's minima
constexpr unsigned kQuadWaveBytes = 2048;
constexpr unsigned kQuadWork = 2 * kBookBytes;
constexpr unsigned kQuadPairs = kQuadWork + kQuadWaves * kQuadWaveBytes;
constexpr unsigned kQuadKeys = kQuadPairs + kQuadWaves * kQuadHeads * 8;
// ROPE: cosines and sines of the lanes' positions for the last kTrigPairs channel pairs; those of the others stay in
// registers, which have no room for all (77 to 134 spilled)
constexpr int kTrigPairs = 24;
constexpr unsigned kQuadTrig(int gh) { return kQuadKeys + 2 * (unsigned)gh * 8; }
constexpr unsigned kQuadLds(int gh, bool rope) { return kQuadTrig(gh) + (rope ? kTrigPairs * 64 * 8 : 0); }
static_assert(kQuadLds(32, true) <= 160 * 1024, "LDS of a CU");
static_assert(kQuadHeads * 128 * 4 == kQuadWaveBytes && kTileTokens * 32 == kQuadWaveBytes, "a wavefront's room");

// minimum over 2^STEPS neighbouring lanes
template <int STEPS>
__device__ __forceinline__ unsigned long long lanes_min_u64(unsigned long long v)
{
    auto smaller = [](unsigned long long k, unsigned lo, unsigned hi) {
        const unsigned long long o = ((unsigned long long)hi << 32) | lo;
        return o < k ? o : k;
    };
    v = smaller(v, dpp_from<0xB1>((unsigned)v), dpp_from<0xB1>((unsigned)(v >> 32)));       // quad_perm [1,0,3,2]
    v = smaller(v, dpp_from<0x4E>((unsigned)v), dpp_from<0x4E>((unsigned)(v >> 32)));       // quad_perm [2,3,0,1]
    v = smaller(v, dpp_from<0x141>((unsigned)v), dpp_from<0x141>((unsigned)(v >> 32)));     // row_half_mirror
    v = smaller(v, dpp_from<0x140>((unsigned)v), dpp_from<0x140>((unsigned)(v >> 32)));     // row_mirror
    if constexpr (STEPS == 5) {
        const auto lo = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((unsigned)(v >> 32), (unsigned)(v >> 32), false, false);
        const unsigned long long a = ((unsigned long long)hi[0] << 32) | lo[0], b = ((unsigned long long)hi[1] << 32) | lo[1];
        v = a < b ? a : b;
    }
    return v;
}

// This lane's and thread's number for what is done once per item (`turn`) at a place (SITE) of the kernel.  ROPE forms them anew:
// kept through the tiles, they and what is derived from them would be spilled, and a spilled register comes back behind
// every load under way.  (The fused step of CQ-8c8b spilled 60, and its first codes were requested when the codebooks had
// arrived: 32 / 8 heads, 8 x 4939 27.5 -> 22.2 us without, 32 x 16384 117.6 -> 112.3.)
struct Place {
    int lane, tid;
};
template <bool ROPE, int SITE>
__device__ __forceinline__ Place place(int turn, int wave)
{
    if constexpr (!ROPE) return Place{(int)threadIdx.x & 63, (int)threadIdx.x};
    unsigned zero;
    asm("v_mov_b32 %0, 0 ; %1 %2" : "=v"(zero) : "s"(turn), "n"(SITE));
    const int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
    return Place{lane, 64 * wave + lane};
}

#define CQ_VIEW_KERNEL 0
#include "cq_decode_quad_kernel.hpp"
#undef CQ_VIEW_KERNEL
#define CQ_VIEW_KERNEL 1
#include "cq_decode_quad_kernel.hpp"
#undef CQ_VIEW_KERNEL

// Neighbouring splits of a call join where that fills the CUs as well: a workgroup walks its items one after the other,
// and every item costs the merge of its wavefronts (about kItemTiles tiles).  Never more partials than the call's split
// has, and decided by sizes alone.  (By ceil(n_split / n), the splits to an item, of which there are about 2 sqrt(n_split): with all n
// a call over 131072 tokens in splits of 64 took 11 us on the host.)
constexpr int kItemTiles = 6;
DecodeArgs joined_splits(const DecodeArgs& a, int n_tiles)
{
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int nh = a.f.n_kv_heads * ((qper + kQuadHeads - 1) / kQuadHeads), resident = nh < 256 ? 256 / nh : 1;
    DecodeArgs best = a;
    int64_t best_cost = -1;
    for (int n = a.n_split; n >= 1;) {
        const int joined = (a.n_split + n - 1) / n, tiles = joined * a.tiles_per_split, split = (n_tiles + tiles - 1) / tiles;
        n = (a.n_split + joined - 1) / joined - 1;
        const int64_t rounds = ((int64_t)a.batch * split + resident - 1) / resident, cost = rounds * (tiles + kItemTiles);
        if (best_cost < 0 || cost < best_cost) {
            best_cost = cost;
            best.tiles_per_split = tiles;
            best.n_split = split;
        }
    }
    return best;
}

template <int GH, int C, bool ROPE, bool STEP, bool LAYERS, int VIEW>
constexpr auto variant()
{
    if constexpr (VIEW == kWhole) return decode_quad_kernel<GH, C, ROPE, STEP, LAYERS>;
    else return decode_quad_view_kernel<GH, C, STEP, VIEW>;
}

template <int GH, int C, bool ROPE, bool STEP, bool LAYERS, int VIEW, class Args>
cq_status launch_variant(const Args& a, const float2* tile_tab, const float2* lane_tab, hipStream_t stream)
{
    constexpr auto kernel = variant<GH, C, ROPE, STEP, LAYERS, VIEW>();
    static LdsKernelSetup setup;
    if (setup.ensure(reinterpret_cast<const void*>(kernel)) != hipSuccess) return CQ_ERR_HIP;
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int nh = a.f.n_kv_heads * ((qper + kQuadHeads - 1) / kQuadHeads);
    const int items = a.batch * a.n_split;
    const int resident = nh < 256 ? 256 / nh : 1;           // one workgroup per CU
    const int per_head = items < resident ? items : resident;
    const unsigned grid = (unsigned)(per_head * nh) * (unsigned)(LAYERS ? a.n_layers : 1);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kQuadThreads), kQuadLds(GH, ROPE), stream, a, tile_tab, lane_tab, items, per_head);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

// (Args: DecodeArgs, or DecodeViewArgs where VIEW is not kWhole)
template <bool ROPE, bool STEP, bool LAYERS, int VIEW = kWhole, class Args = DecodeArgs>
cq_status launch_format(const Args& a, const float2* tile_tab, const float2* lane_tab, hipStream_t stream)
{
    if (a.f.b != 8 || a.f.head_dim != 128) return CQ_ERR_UNSUPPORTED;
    if (a.f.c == 8) return launch_variant<16, 8, ROPE, STEP, LAYERS, VIEW>(a, tile_tab, lane_tab, stream);
    if (a.f.c == 4) return launch_variant<32, 4, ROPE, STEP, LAYERS, VIEW>(a, tile_tab, lane_tab, stream);
    return CQ_ERR_UNSUPPORTED;
}

}  // namespace

// Whether a call over keys as stored goes here rather than to the kernels with tables and bins (cq_decode.hip, cq_decode_pair.hip):
// query heads in fours, enough items for the CUs (one workgroup each, 256), and, of CQ-8c8b, splits that are short or
// fill their rounds; 32 / 8 heads, tables -> here, us per cq_decode_attention call:
//   CQ-4c8b  18 x 64 11.6 -> 7.0, 64 x 64 31.4 -> 9.7, 64 x 300 32.6 -> 11.9, 18 x 1100 17.1 -> 10.5, 64 x 1100 41.3 -> 18.6, 20 x 2000 20.9 -> 13.4,
//            12 x 8000 (two splits) 31.4 -> 22.9, 34 x 4200 49.0 -> 38.1, 48 x 16000 131 -> 116, 64 x 16000 189 -> 131; with 128 items (16
//            sequences, which fill the CUs in pairs) 300 9.1 -> 7.7, 2000 13.2 -> 13.4, 4200 18.0 -> 20.7, 16000 46.9 -> 58.7
//   CQ-8c8b  18 x 64 10.5 -> 7.1, 64 x 64 31.3 -> 8.7, 64 x 300 31.8 -> 10.9, 18 x 1100 13.0 -> 10.1, 64 x 1100 36.0 -> 17.1, 20 x 4200 22.2 -> 19.3,
//            28 x 4200 27.4 -> 19.5, 64 x 16000 123 -> 105; 128 items: 300 9.0 -> 7.2, 2000 10.9 -> 12.1
// (the fused step, with its search here, alike: 18 x 64 17.4 -> 9.6 and 15.4 -> 8.8, 34 x 2000 39.6 -> 27.9 and 29.8 -> 25.4).
// A tile of CQ-8c8b costs 434 clocks of the LDS here and 258 with tables, so long splits, as they are walked here (joined), have
// to fill their rounds: of 250 tiles 18 / 20 / 24 x 16000 50.7 / 51.7 / 51.7 -> 53.6 / 53.3 / 53.1, 28 x 16000 61.8 -> 54.1; of 125 tiles 18 x
// 8000 30.3 -> 30.1, 12 x 16000 33.0 -> 33.0; in two rounds 34 x 8000 46.3 -> 56.7, 34 x 4200 33.6 -> 34.7, 34 x 2000 21.8 -> 20.8.  One of
// CQ-4c8b costs 476 and 515.
bool decode_takes_quads(const DecodeArgs& a, int n_tiles, DecodeArgs* joined)
{
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    if (a.f.b != 8 || a.f.c < 4 || a.f.head_dim != 128 || qper % kQuadHeads != 0) return false;
    const int64_t items_per_split = (int64_t)a.batch * (a.n_q_heads / kQuadHeads);
    if (items_per_split * a.n_split < 140) return false;
    const DecodeArgs j = joined_splits(a, n_tiles);
    const int64_t items = items_per_split * j.n_split, rounds = (items + 255) / 256;
    if (items < 140) return false;
    *joined = j;
    if (a.f.c == 4) return true;
    return items * 100 >= rounds * 256 * 78 || j.tiles_per_split <= (rounds == 1 ? 128 : 64);
}

cq_status launch_decode_quad(const DecodeArgs& a, hipStream_t stream)
{
    const cq_status st = a.layers   ? launch_format<false, true, true>(a, nullptr, nullptr, stream)
                         : a.xk_new ? launch_format<false, true, false>(a, nullptr, nullptr, stream)
                                    : launch_format<false, false, false>(a, nullptr, nullptr, stream);
    if (st != CQ_OK || a.n_split == 1) return st;
    return launch_decode_merge(a, stream);
}

cq_status launch_decode_quad_view(const DecodeViewArgs& a, hipStream_t stream)
{
    const cq_status st = a.scores   ? launch_format<false, false, false, kScores>(a, nullptr, nullptr, stream)
                         : a.xk_new ? launch_format<false, true, false, kWindow>(a, nullptr, nullptr, stream)
                                    : launch_format<false, false, false, kWindow>(a, nullptr, nullptr, stream);
    if (st == CQ_OK && a.scores) return launch_decode_weights(a, stream);
    if (st != CQ_OK || a.n_split == 1) return st;
    return launch_decode_merge(a, stream);
}

cq_status launch_decode_quad_rope(const DecodeArgs& a_in, const float2* tile_tab, const float2* lane_tab, hipStream_t stream)
{
    // (every call of grouped queries comes here, and a given split fixes its bits in any batch: joining, which follows the
    // batch, is for the library's own split)
    const DecodeArgs a = a_in.split_given ? a_in : joined_splits(a_in, (a_in.t + kTileTokens - 1) / kTileTokens);
    const cq_status st = a.xk_new ? launch_format<true, true, false>(a, tile_tab, lane_tab, stream) : launch_format<true, false, false>(a, tile_tab, lane_tab, stream);
    if (st != CQ_OK || a.n_split == 1) return st;
    return launch_decode_merge(a, stream);
}

}  // namespace cq
