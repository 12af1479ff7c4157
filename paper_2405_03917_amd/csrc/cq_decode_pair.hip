// Decode attention straight from packed CQ codes for grouped queries: a workgroup of 16 wavefronts serves TWO
// query heads of a KV head (cq_decode.hip: one, and what the kernels have in common), for gfx950.
//
// What bounds grouped queries is not the code streams, which further heads of a KV head find in L2, but the LDS: a
// gather and an add per group, token and head.  The LDS reads 64 bits per lane in the time of 32 (measured, clocks
// per wavefront and CU without bank conflicts: ds_read_b32 and ds_read_b64 2.05, ds_read_b128 4.1, ds_add_u32 4.0,
// ds_add_u64 6.0), so a cell of the score table and of the bins is a pair of words here, one per head: 8.1 clocks
// for a gather and an add of both heads against 12.2, and the codes, their addresses, the codebooks and the new
// token's search are shared.  (A group of four heads would take ds_read_b128 and two ds_add_u64: as many LDS clocks per head.)
// Table and bins of CQ-8c8b and CQ-4c8b are 64 KB each (SEPARATE), those of CQ-2c8b and CQ-8c10b share 128 KB
// (SHARED): one workgroup has the CU, and nothing overlaps its table build and epilogue.
//
// Measured (32 / 8 heads; one head per workgroup -> two, both with the present kernels on one card): CQ-8c10b, batch 32 x 16384
// 103.6 -> 77.6 us (74 to 78 on other cards), its step 132.8 -> 92.4, batch 16 x 300 16.3 -> 12.2; CQ-2c8b, batch 16 x 4096
// 37.2 -> 29.5; CQ-4c8b, 32 x 16384 115.5 -> 94.0, 16 x 4096 20.3 -> 17.1; CQ-8c8b, 32 x 16384 66.2 -> 62.9.  The walk's key half is bound by the vector ALU (about 220 clocks per tile and SIMD
// against 33 of LDS per CU), its value half by the LDS (96 per CU against 170 of vector ALU per SIMD), and all wavefronts are in
// the same half.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cq_decode_split.hpp"

namespace cq {
namespace {

constexpr int H = 2;                                    // query heads of a workgroup
constexpr int kPairThreads = kDecodeThreads * H;

// ---- layout of the workgroup's LDS
template <int GH, int B>
struct Lay {
    static constexpr int K = 1 << B;
    static constexpr int NW = kDecodeWaves * H;                     // wavefronts
    static constexpr bool SEPARATE = B == 8 && GH <= 32;            // table and bins side by side (else one after the other)
    static constexpr int R = (GH == 16 && B == 8) ? 2 : 1;          // replicas per group
    static constexpr unsigned TAB_BYTES = 131072;                   // table and bins
    static constexpr unsigned BIN_BYTES = SEPARATE ? 65536 : 0;     // the bins' cells, this far behind the table's
    static constexpr int ROW_BYTES = SEPARATE ? 256 : 512;
    static constexpr int TILE_BYTES = kTileTokens * GH * B / 8;
    static constexpr int SLOTS = TAB_BYTES / 4;                     // [2][H][2][NW] floats
    static constexpr int SUMS = SLOTS + 4 * H * NW;                 // [H][NW] unsigned
    static constexpr int SCR = SUMS + H * NW;                       // 64 + H * NW * head_dim floats
    static constexpr int KEYS(int head_dim) { return SCR + 64 + H * NW * head_dim; }   // fused step only
    // fused step: the keys, the new token's fixed-point weights, its record of key codes in cache order
    static constexpr int FLOATS(int head_dim, bool step) { return KEYS(head_dim) + (step ? NewTokenWords<GH, B>::END : 0); }
    // Byte address of the cell of code value j in column `col`.  b = 8: row j.  b = 10: row = the low 8 bits,
    // and the two high bits pick one of four 16-cell quarters of the row.
    __device__ __forceinline__ static constexpr unsigned cell(int j, int col)
    {
        return B == 8 ? (unsigned)(j * ROW_BYTES + col * 8) : (unsigned)((j & 255) * ROW_BYTES + (j >> 8) * 128 + col * 8);
    }
};

// Per-lane column constants for the Gh slots of a token, four byte offsets per register: of 8-byte columns
// (SEPARATE), or of 4-byte columns, doubled together with the code (SHARED: rows of 512 bytes).
template <int GH, int B>
struct Cols {
    unsigned v[GH / 4];
    __device__ __forceinline__ void init(int lane)
    {
#pragma unroll
        for (int i = 0; i < GH / 4; ++i) {
            unsigned x = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int g = (lane + 4 * i + k) & (GH - 1);
                const int column = Lay<GH, B>::R == 2 ? 2 * g + ((lane >> 4) & 1) : g;   // lanes l and l + 16 differ, l and l + 32 share
                x |= (unsigned)((Lay<GH, B>::SEPARATE ? 8 : 4) * column) << (8 * k);
            }
            v[i] = x;
        }
    }
};

// Byte address of the cell for slot s of this lane's token, of the table or (BIN) of the bins.  (The bins of SEPARATE
// are 64 KB further, one more than an LDS instruction's offset field holds.)
template <bool BIN, int GH, int B>
__device__ __forceinline__ unsigned code_addr(const Tile<GH, B>& w, const Cols<GH, B>& col, int s)
{
    const u32x4 q = w.lo[s >> 4];
    const int dw = (s >> 2) & 3;
    const unsigned code_word = dw == 0 ? q.x : dw == 1 ? q.y : dw == 2 ? q.z : q.w;
    const unsigned k = s & 3;
    const unsigned sel = 0x0c0c0000u | ((4u + k) << 8) | k;   // {0, 0, code byte k, column byte k}
    unsigned at = __builtin_amdgcn_perm(code_word, col.v[s >> 2], sel);
    if constexpr (B != 8) at |= ((w.hi >> (2 * s)) & 3u) << 6;
    if constexpr (!Lay<GH, B>::SEPARATE) at <<= 1;
    if constexpr (BIN) at |= Lay<GH, B>::BIN_BYTES;
    return at;
}

typedef float pair_f32 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) pair_f32 lds_pair;
typedef __attribute__((address_space(3))) unsigned long long lds_u64;

// (phases, fixed point, the fused step and the walk as in the kernel for one head; m0, l, fx, ... are kept per head)
#define CQ_VIEW_KERNEL 0
#include "cq_decode_pair_kernel.hpp"
#undef CQ_VIEW_KERNEL
#define CQ_VIEW_KERNEL 1
#include "cq_decode_pair_kernel.hpp"
#undef CQ_VIEW_KERNEL

template <int GH, int C, int B, int NS, bool STEP, bool LAYERS, int VIEW>
constexpr auto variant()
{
    if constexpr (VIEW == kWhole) return decode_pair_kernel<GH, C, B, NS, STEP, LAYERS>;
    else return decode_pair_view_kernel<GH, C, B, NS, STEP, VIEW>;
}

template <int GH, int C, int B, int NS, bool STEP, bool LAYERS, int VIEW, class Args>
cq_status launch_variant(const Args& a, hipStream_t stream)
{
    constexpr auto kernel = variant<GH, C, B, NS, STEP, LAYERS, VIEW>();
    static LdsKernelSetup setup;
    if (setup.ensure(reinterpret_cast<const void*>(kernel)) != hipSuccess) return CQ_ERR_HIP;
    using F = Lay<GH, B>;
    if (!F::SEPARATE && a.tiles_per_split > NS * F::NW) return CQ_ERR_INVALID_ARG;
    const size_t smem = sizeof(float) * (size_t)F::FLOATS(a.f.head_dim, STEP);
    if (smem > 160 * 1024) return CQ_ERR_INVALID_ARG;
    const unsigned grid = (unsigned)(a.batch * (a.n_q_heads / H) * a.n_split) * (unsigned)(a.layers ? a.n_layers : 1);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kPairThreads), smem, stream, a);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

template <int GH, int C, int B, int NS, bool STEP, bool LAYERS, int VIEW, class Args>
cq_status launch_by_length(const Args& a, hipStream_t stream)
{
    if (decode_pair_chunk_tiles(a) == NS / 4) return launch_variant<GH, C, B, NS / 4, STEP, LAYERS, VIEW>(a, stream);
    return launch_variant<GH, C, B, NS / 2, STEP, LAYERS, VIEW>(a, stream);
}

// (Args: DecodeArgs, or DecodeViewArgs where VIEW is not kWhole)
template <bool STEP, bool LAYERS, int VIEW = kWhole, class Args = DecodeArgs>
cq_status launch_format(const Args& a, hipStream_t stream)
{
    if (a.f.b == 8) {
        if (a.f.gh == 16 && a.f.c == 8) return launch_by_length<16, 8, 8, kChunkTiles8, STEP, LAYERS, VIEW>(a, stream);
        if (a.f.gh == 32 && a.f.c == 4) return launch_by_length<32, 4, 8, kChunkTiles8, STEP, LAYERS, VIEW>(a, stream);
        if (a.f.gh == 64 && a.f.c == 2) return launch_by_length<64, 2, 8, kChunkTiles8, STEP, LAYERS, VIEW>(a, stream);
    } else if (a.f.b == 10 && a.f.gh == 16 && a.f.c == 8) {
        return launch_by_length<16, 8, 10, kChunkTiles10, STEP, LAYERS, VIEW>(a, stream);
    }
    return CQ_ERR_UNSUPPORTED;
}

}  // namespace

// An even number of query heads per KV head, and enough workgroups: one runs per CU, so fewer than 256 leave CUs idle
// that the kernel for one head uses, and with byte codes a last round of workgroups that fills less than its share
// costs more than the pairs save (32 / 8 heads, one head -> two: 1.25 rounds, 20 x 2000, CQ-8c8b 14.7 -> 19.9 us, CQ-4c8b 20.8 ->
// 24.0; 1.5 rounds, 24 x 3000, step of CQ-4c8b 30.9 -> 33.7; 1.75 rounds, 28 x 4000, CQ-8c8b 25.2 -> 25.4, CQ-4c8b 37.8 -> 32.7, and 28 x
// 16000 64.9 -> 62.4, 110.7 -> 91.6).  CQ-8c10b gains in nearly all of them (17 x 2000 28.0 -> 29.1, 17 x 16000 76.5 -> 71.6, 20 x 2000 28.9 ->
// 29.4, 20 x 16000 78.2 -> 72.0, 24 x 2000 30.3 -> 29.7, 36 x 2000 45.4 -> 43.5): of its codebooks, 256 KB each, a workgroup reads
// half as much per head.  (Calls of CQ-8c8b and CQ-4c8b with heads in fours are offered to cq_decode_quad.hip first, which takes those
// byte-code sizes above; the rule is for two or six heads per KV head as it was for four.  Of a layer-batched launch the layer
// decides, so that its results are those of the layers' own calls.)
bool decode_takes_pairs(const DecodeArgs& a)
{
    const int qper = a.n_q_heads / a.f.n_kv_heads;
    const int64_t wgs = (int64_t)a.batch * (a.n_q_heads / H) * a.n_split, rounds = (wgs + 255) / 256;
    if (qper % H != 0 || wgs < 256) return false;
    return a.f.b == 10 || wgs * 20 >= rounds * 256 * 17;
}

// (twice the wavefronts: half the tiles per wavefront and chunk, of two heads each, so as many score registers)
int decode_pair_chunk_tiles(const DecodeArgs& a)
{
    const int full = (a.f.b == 10 ? kChunkTiles10 : kChunkTiles8) / H, nw = kDecodeWaves * H;
    return (a.tiles_per_split + nw - 1) / nw <= full / 2 ? full / 2 : full;
}

cq_status launch_decode_pair(const DecodeArgs& a, hipStream_t stream)
{
    if (a.layers) return launch_format<true, true>(a, stream);
    return a.xk_new ? launch_format<true, false>(a, stream) : launch_format<false, false>(a, stream);
}

cq_status launch_decode_pair_view(const DecodeViewArgs& a, hipStream_t stream)
{
    if (a.scores) return launch_format<false, false, kScores>(a, stream);
    return a.xk_new ? launch_format<true, false, kWindow>(a, stream) : launch_format<false, false, kWindow>(a, stream);
}

}  // namespace cq
