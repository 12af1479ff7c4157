// Decode attention straight from packed CQ codes (Eq. 1 of the paper over the centroids the
// cached codes select), for gfx950.
//
// One workgroup handles one (sequence, query head, context split).  Per workgroup:
//   1. build the score table  LUT[g][j] = scale * log2(e) * (q_g . C_K[g][j])  in LDS;
//   2. walk the split chunk by chunk (a chunk is 16 tiles of 64 tokens per wavefront):
//      K: stream the chunk's key codes (one tile per wavefront per step, lane = token),
//         score = sum over groups of LUT[g][code]; the scores stay in registers;
//      V: stream the chunk's value codes; p = 2^(score - reference) in fixed point; add p into
//         bin[g][code] in LDS with integer atomics (exact, order independent);
//   3. epilogue: o[g c + i] = sum_j bin[g][j] * C_V[g][j][i]; with a single split the normalised
//      result is rounded to fp16 and stored, otherwise (max, sum p, o) goes out as a partial and
//      a second kernel merges the partials of all splits.
//
// LDS table layout: 256 rows of 64 four-byte words (64 KB); b = 8: one row per code value;
// b = 10: one row per value of a code's low byte, whose four 16-word quarters belong to the
// four values of its two high bits.  Lane l of a wavefront owns ONE word
// column at every step s of the walk over a token's Gh slots: column(l, g) with g = (l + s) mod
// Gh, the group that the cache layout put in slot s of token l.  With 32 or 64 groups per head
// the 32 columns of a half-wavefront are different modulo 32 (lanes l and l + 32 may share one:
// the LDS serves a wavefront in two halves), so neither the table gather nor the bin update ever
// has a bank conflict.  With 16 groups per head and b = 8 each group is replicated twice to give
// 32 lanes their own column (the epilogue adds the replicas); b = 10 keeps one column per
// group.  For b = 8 the byte address of a lookup is (code << 8) | (4 * column): one v_perm_b32
// from the code word and a per-lane constant; b = 10 ors the two high bits in behind it.  With 16 or 32 groups per head words 0..31 of a
// 256-byte row are the table's columns and words 32..63 the bins', so both exist at once and a
// workgroup can walk any number of chunks with one table; 64 groups per head and b = 10 turn the
// table into the bins once their single chunk is scored.  Every format needs 70 KB of LDS, so
// two workgroups share a CU.
//
// Measured on MI355X (microbenchmark, per CU): ds_read_b32 gathers and ds_add_u32 run at the
// same rate with this layout as with linear addresses; ds_add_f32 is about 45 times slower than
// ds_add_u32, which is why the bins are integers.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cq_decode_split.hpp"

// arrival counters of the in-kernel merge (see MergeCounters); 512 KB per GPU
static __device__ __align__(256) unsigned merge_counters[16 * 8192];

namespace cq {
namespace {

// Tiles per wavefront of the shortest splits (see ONCE), 2048 tokens of CQ-8c8b: batch 1 x 2000, 32 heads 8.95 -> 8.68 us, its
// step 10.9 -> 10.5; step of batch 2 x 1000 9.6 -> 9.0.  None for the other formats: their codebook is walked in two and
// four parts, which the tiles' requests then hold up (CQ-4c8b, batch 16 x 900: 12.4 -> 13.2), and CQ-2c8b has no registers left.
// Layer-batched launches have no such form yet, for no other reason than that it was not built with it: theirs would gain too
// (cq_decode_step_layers, 32 layers of batch 1 x 1000 33.7 -> 31.5 us, 1 x 2000 54.5 -> 49.4, 8 x 1000 195 -> 150).
constexpr int kOnceTiles(int gh) { return gh == 16 ? 4 : 0; }
constexpr int kMergeRows = 8192;        // arrival counters per set (rows of one launch)
constexpr int kMergeSets = 16;          // sets (streams served) per device
static_assert(sizeof(merge_counters) == sizeof(unsigned) * kMergeRows * kMergeSets, "size of the counter array");

__global__ void layer_table_write_kernel(LayerChunk chunk, int count, LayerPtrs* dst)
{
    if ((int)threadIdx.x < count) dst[threadIdx.x] = chunk.p[threadIdx.x];
}

// A kernel argument is loaded (scalar load from the argument block) where it is first used;
// left to the compiler, the prologue of this kernel loads its arguments in four dependent
// stages (head counts; split and context; strides; pointers), each awaited before the next is
// requested, and an argument added to a late stage delays the first global load (measured: 0.3-0.4
// us per launch of the attention kernel for two more strides).  early() pins a value in a scalar
// register at the point of the call, so that everything the workgroup needs before its first
// global load is requested together at entry and awaited once.
// (A pointer comes back as a pointer into global memory, which is what every pointer argument
// of these kernels is: a pointer of unknown provenance would make each access through it a flat
// instruction.)
template <class T>
__device__ __forceinline__ T* early(T* p)
{
    unsigned long long x = reinterpret_cast<unsigned long long>(p);
    asm volatile("" : "+s"(x));
    return (T*)reinterpret_cast<__attribute__((address_space(1))) T*>(x);
}
template <class T>
__device__ __forceinline__ T early(T v)
{
    if constexpr (sizeof(T) == 4) {
        unsigned x = __builtin_bit_cast(unsigned, v);
        asm volatile("" : "+s"(x));
        return __builtin_bit_cast(T, x);
    } else {
        static_assert(sizeof(T) == 8, "32- or 64-bit arguments");
        unsigned long long x = __builtin_bit_cast(unsigned long long, v);
        asm volatile("" : "+s"(x));
        return __builtin_bit_cast(T, x);
    }
}

template <bool STEP, bool LAYERS, class Args>
__device__ __forceinline__ Args early_args(const Args& in)
{
    Args a = in;                  // (what is not named below is read where it is used)
    // (not for a layer-batched launch: its workgroups overlap one another's prologues anyway, and
    // the pinned registers cost that variant 2 % at 32 groups per head)
    if constexpr (LAYERS) return a;
    a.n_q_heads = early(in.n_q_heads);
    a.f.n_kv_heads = early(in.f.n_kv_heads);
    a.n_split = early(in.n_split);
    a.tiles_per_split = early(in.tiles_per_split);
    a.t = early(in.t);
    a.seq_lens = early(in.seq_lens);
    a.seq_len_shift = early(in.seq_len_shift);
    a.seq_len_floor = early(in.seq_len_floor);
    a.map.block_table = early(in.map.block_table);
    a.map.bt_stride = early(in.map.bt_stride);
    a.map.n_pages = early(in.map.n_pages);
    a.map.tiles_cap = early(in.map.tiles_cap);
    a.map.n_kv_heads = early(in.map.n_kv_heads);
    a.scale_log2e = early(in.scale_log2e);
    a.partials = early(in.partials);
    a.q = early(in.q);
    a.k_codes = early(in.k_codes);
    a.v_codes = early(in.v_codes);
    a.k_centroids = early(in.k_centroids);
    a.v_centroids = early(in.v_centroids);
    a.out = early(in.out);
    a.q_batch_stride = early(in.q_batch_stride);
    a.out_batch_stride = early(in.out_batch_stride);
    if constexpr (STEP) {
        a.xk_new = early(in.xk_new);
        a.xv_new = early(in.xv_new);
        a.x_new_stride = early(in.x_new_stride);
    }
    return a;
}

// ---- layout of the workgroup's LDS ---------------------------------------------------------
// b = 8, 16 or 32 groups per head (SEPARATE): every 256-byte row holds the score table in words
// 0..31 and the probability bins in words 32..63 (16 groups per head: two replicas of each, so
// that the 32 lanes of a half-wavefront own 32 different banks), 64 KB in all.  Table and bins
// live side by side, so a workgroup can walk a context of any length chunk by chunk with the
// table it built once.
// b = 8 with 64 groups per head, b = 10 (SHARED): the table fills the 64 KB; it is cleared after
// the scores of the (single) chunk are known and becomes the bins.
// Behind the table: the wavefronts' (maximum, sum) pairs of a chunk (two sets, used alternately),
// their integer sums at a rescale, the reduction scratch of the epilogue, the fused step's keys.
template <int GH, int B>
struct Lay {
    static constexpr int K = 1 << B;
    static constexpr int RW = 64;                                   // words per row
    static constexpr bool SEPARATE = B == 8 && GH <= 32;
    static constexpr int R = (GH == 16 && B == 8) ? 2 : 1;          // replicas per group
    static constexpr int BIN0 = SEPARATE ? 32 : 0;                  // first bin word of a row
    static constexpr int TAB_FLOATS = 256 * RW;
    static constexpr int TILE_BYTES = kTileTokens * GH * B / 8;
    static constexpr int SLOTS = TAB_FLOATS;                        // [2][2][NW] floats
    static constexpr int SUMS = SLOTS + 4 * kDecodeWaves;           // [NW] unsigned
    static constexpr int SCR = SUMS + kDecodeWaves;                 // 64 + NW * head_dim floats
    static constexpr int KEYS(int head_dim) { return SCR + 64 + kDecodeWaves * head_dim; }   // fused step only
    // fused step: the keys, the new token's fixed-point weight, its record of key codes in cache order
    static constexpr int FLOATS(int head_dim, bool step) { return KEYS(head_dim) + (step ? NewTokenWords<GH, B>::END : 0); }
    // Word of code value j in word column `col`.  b = 8: row j.  b = 10: row = the low 8 bits,
    // and the two high bits pick one of four 16-word quarters of the row, which makes the byte
    // address (low << 8) | (high << 6) | (4 * column): the b = 8 address plus one shift-or.
    __device__ __forceinline__ static constexpr int word(int j, int col)
    {
        return B == 8 ? j * 64 + col : (j & 255) * 64 + (j >> 8) * 16 + col;
    }
};

// Per-lane column constants for the Gh slots of a token, four byte offsets per register (the
// table's columns; the bins' are Lay::BIN0 words further, which rides in the offset field of
// the LDS instruction).
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
                x |= (unsigned)(4 * column) << (8 * k);
            }
            v[i] = x;
        }
    }
};

// Byte address of the word for slot s of this lane's token.
template <int GH, int B>
__device__ __forceinline__ unsigned code_addr(const Tile<GH, B>& w, const Cols<GH, B>& col, int s)
{
    const u32x4 q = w.lo[s >> 4];
    const int dw = (s >> 2) & 3;
    const unsigned code_word = dw == 0 ? q.x : dw == 1 ? q.y : dw == 2 ? q.z : q.w;
    const unsigned k = s & 3;
    const unsigned sel = 0x0c0c0000u | ((4u + k) << 8) | k;   // {0, 0, code byte k, column byte k}
    const unsigned lo = __builtin_amdgcn_perm(code_word, col.v[s >> 2], sel);
    if constexpr (B == 8) return lo;
    else return (((w.hi >> (2 * s)) & 3u) << 6) | lo;
}

// STEP = true is the fused decode step: the workgroup whose split holds the newest position
// (t_n - 1) also encodes that token's key and value rows for its KV head.  Keys: while it builds
// the score table (the key codebook is in registers anyway); the tile that holds the position is
// then patched in registers as if the codes were already in the cache.  Values: in the epilogue
// (the value codebook is in registers there); phase V leaves the position out of the bins and
// its weight is added to the bins of the codes just found.  The first query head of each KV head
// stores the codes.  Results equal cq_encode_kv followed by cq_decode_attention bit for bit
// (the bins are integers: the order of the additions does not matter).
//
// The walk.  Wavefront w owns tiles w, w + 8, ... of the split; a CHUNK is NS of its tiles (8 NS
// tiles of the workgroup).  Per chunk: the key tiles give one score per lane and tile, kept in
// NS registers (lane = token in both streams, so the lane that scored a token also bins it);
// the wavefronts exchange the chunk's (maximum, sum of 2^(score - maximum)) across one barrier;
// then the value tiles are binned.  Requests run PF tiles ahead through both streams and across
// chunk boundaries.
#define CQ_VIEW_KERNEL 0
#include "cq_decode_split_kernel.hpp"
#undef CQ_VIEW_KERNEL
#define CQ_VIEW_KERNEL 1
#include "cq_decode_split_kernel.hpp"
#undef CQ_VIEW_KERNEL

// Merge the partials of all splits of one (sequence, query head): rescaling to the running
// maximum split by split, then one rounding to fp16.
__global__ void decode_merge_kernel(const float* partials, uint16_t* out, int n_split, int head_dim,
                                    const LayerPtrs* layers, int rows_per_layer, int n_q_heads, int64_t out_batch_stride)
{
    int bh = blockIdx.x;
    const int stride = head_dim + kPartialHeader;
    const float* p = partials + (size_t)bh * n_split * stride;
    if (layers) {                       // layer-batched: row bh of layer blockIdx / rows_per_layer
        const int layer = bh / rows_per_layer;
        bh -= layer * rows_per_layer;
        out = layers[layer].out;
    }
    out += (size_t)(bh / n_q_heads) * out_batch_stride + (size_t)(bh % n_q_heads) * head_dim;
    merge_splits<false>(p, n_split, head_dim, out, threadIdx.x, blockDim.x);
}

// Arrival counters of the in-kernel merge: one per (sequence, query head) row of a launch.  They
// start at zero (static storage) and every launch leaves them at zero, so they need no clearing;
// what they need is that no two launches that can overlap share a set.  Launches on one stream
// never overlap, so every stream gets a set of its own (the first kMergeSets streams that ask,
// per device; a stream keeps its set).  A stream under graph capture gets none: replays of its
// graph may run on other streams, at the same time as one another.  Whoever gets no set runs
// the separate merge kernel instead.
struct MergeCounters {
    static constexpr int kMaxDevices = 64;
    struct PerDevice {
        std::mutex mu;
        unsigned* base = nullptr;
        bool failed = false;
        hipStream_t streams[kMergeSets];
        int n = 0;
    };
    PerDevice dev[kMaxDevices];

    unsigned* for_stream(hipStream_t stream, int rows)
    {
        if (rows > kMergeRows) return nullptr;
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        if (hipStreamIsCapturing(stream, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) {
            (void)hipGetLastError();
            return nullptr;
        }
        int d = 0;
        if (hipGetDevice(&d) != hipSuccess || d < 0 || d >= kMaxDevices) return nullptr;
        PerDevice& pd = dev[d];
        std::lock_guard<std::mutex> lock(pd.mu);
        if (pd.failed) return nullptr;
        if (!pd.base) {
            void* p = nullptr;
            if (hipGetSymbolAddress(&p, HIP_SYMBOL(merge_counters)) != hipSuccess || !p) {
                pd.failed = true;
                return nullptr;
            }
            pd.base = static_cast<unsigned*>(p);
        }
        for (int i = 0; i < pd.n; ++i)
            if (pd.streams[i] == stream) return pd.base + (size_t)i * kMergeRows;
        if (pd.n == kMergeSets) return nullptr;
        pd.streams[pd.n] = stream;
        return pd.base + (size_t)(pd.n++) * kMergeRows;
    }
};
MergeCounters g_merge_counters;

template <int GH, int C, int B, int NS, bool STEP, bool LAYERS, int VIEW>
constexpr auto variant()
{
    if constexpr (VIEW == kWhole) return decode_split_kernel<GH, C, B, NS, STEP, LAYERS>;
    else return decode_split_view_kernel<GH, C, B, NS, STEP, VIEW>;
}

template <int GH, int C, int B, int NS, bool STEP, bool LAYERS, int VIEW, class Args>
cq_status launch_variant(const Args& a, hipStream_t stream)
{
    constexpr auto kernel = variant<GH, C, B, NS, STEP, LAYERS, VIEW>();
    static LdsKernelSetup setup;
    if (setup.ensure(reinterpret_cast<const void*>(kernel)) != hipSuccess) return CQ_ERR_HIP;
    using F = Lay<GH, B>;
    if (!F::SEPARATE && a.tiles_per_split > NS * kDecodeWaves) return CQ_ERR_INVALID_ARG;
    const size_t smem = sizeof(float) * (size_t)F::FLOATS(a.f.head_dim, STEP);
    if (smem > 160 * 1024) return CQ_ERR_INVALID_ARG;
    const unsigned grid = (unsigned)(a.batch * a.n_q_heads * a.n_split) * (unsigned)(a.layers ? a.n_layers : 1);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kDecodeThreads), smem, stream, a);
    if (hipGetLastError() != hipSuccess) return CQ_ERR_HIP;
    return CQ_OK;
}

// tiles per wavefront and chunk that a call's splits take
int chunk_tiles(const DecodeArgs& a)
{
    const int full = a.f.b == 10 ? kChunkTiles10 : kChunkTiles8;
    const int tiles_per_wave = (a.tiles_per_split + kDecodeWaves - 1) / kDecodeWaves;
    if (a.f.b == 8 && !a.layers && tiles_per_wave <= kOnceTiles(a.f.gh)) return kOnceTiles(a.f.gh);
    return tiles_per_wave <= full / 2 ? full / 2 : full;
}

template <int GH, int C, int B, int NS, bool STEP, bool LAYERS, int VIEW, class Args>
cq_status launch_by_length(const Args& a, hipStream_t stream)
{
    const int ns = chunk_tiles(a);
    if constexpr (B == 8 && !LAYERS && kOnceTiles(GH) > 0) {
        if (ns == kOnceTiles(GH)) return launch_variant<GH, C, B, kOnceTiles(GH), STEP, LAYERS, VIEW>(a, stream);
    }
    if (ns == NS / 2) return launch_variant<GH, C, B, NS / 2, STEP, LAYERS, VIEW>(a, stream);
    return launch_variant<GH, C, B, NS, STEP, LAYERS, VIEW>(a, stream);
}

// (Args: DecodeArgs, or DecodeViewArgs where VIEW is not kWhole)
template <bool STEP, bool LAYERS, int VIEW = kWhole, class Args = DecodeArgs>
cq_status launch_format(const Args& a, hipStream_t stream)
{
    // 70 KB of LDS per workgroup in every format: two 512-thread workgroups share a CU
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

cq_status launch_layer_table_write(const LayerChunk& chunk, int count, LayerPtrs* dst, hipStream_t stream)
{
    hipLaunchKernelGGL(layer_table_write_kernel, dim3(1), dim3(64), 0, stream, chunk, count, dst);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

cq_status launch_decode_merge(const DecodeArgs& a, hipStream_t stream)
{
    const int rows = a.batch * a.n_q_heads;
    hipLaunchKernelGGL(decode_merge_kernel, dim3((unsigned)(rows * (a.layers ? a.n_layers : 1))), dim3(128), 0, stream,
                       a.partials, a.out, a.n_split, a.f.head_dim, a.layers, rows, a.n_q_heads, a.out_batch_stride);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

cq_status launch_decode_merge(const float* partials, uint16_t* out, int rows, int n_q_heads, int64_t out_batch_stride,
                              int n_split, int head_dim, hipStream_t stream)
{
    hipLaunchKernelGGL(decode_merge_kernel, dim3((unsigned)rows), dim3(128), 0, stream, partials, out, n_split, head_dim,
                       static_cast<const LayerPtrs*>(nullptr), 0, n_q_heads, out_batch_stride);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

int decode_max_tiles_per_split(const Derived& f)
{
    // formats whose table and bins share their LDS walk one chunk per workgroup; the others walk
    // any number of chunks (the bound below only keeps the index arithmetic inside 32 bits)
    if (f.b == 10) return kChunkTiles10 * kDecodeWaves;                // 16384 tokens
    if (f.gh == 64) return kChunkTiles8 * kDecodeWaves;                // 8192 tokens
    return 1 << 20;
}

DecodePlan decode_plan(const DecodeArgs& a)
{
    DecodeArgs joined;
    if (decode_takes_quads(a, (a.t + kTileTokens - 1) / kTileTokens, &joined)) return DecodePlan{4, 1};
    return decode_takes_pairs(a) ? DecodePlan{2, decode_pair_chunk_tiles(a)} : DecodePlan{1, chunk_tiles(a)};
}

cq_status launch_decode(const DecodeArgs& a_in, hipStream_t stream)
{
    DecodeArgs a;
    if (decode_takes_quads(a_in, (a_in.t + kTileTokens - 1) / kTileTokens, &a)) return launch_decode_quad(a, stream);
    a = a_in;
    a.merge_counters = a.n_split > 1 ? g_merge_counters.for_stream(stream, a.batch * a.n_q_heads * (a.layers ? a.n_layers : 1)) : nullptr;
    // (a layer-batched launch is always a fused step: its table holds the new rows)
    const cq_status st = decode_takes_pairs(a) ? launch_decode_pair(a, stream)
                         : a.layers ? launch_format<true, true>(a, stream) : a.xk_new ? launch_format<true, false>(a, stream) : launch_format<false, false>(a, stream);
    if (st != CQ_OK || a.n_split == 1 || a.merge_counters) return st;
    return launch_decode_merge(a, stream);
}

cq_status launch_decode_view(const DecodeViewArgs& a_in, hipStream_t stream)
{
    DecodeViewArgs a = a_in;
    if (decode_takes_quads(a_in, view_tiles(a_in.t, 1, a_in.window, a_in.n_sink), &a)) return launch_decode_quad_view(a, stream);
    // With the scores kept, the weights need all splits of a row and all query heads of a KV head.  One query head and a short
    // context: the row's last workgroup adds them up as it merges the output; so, too, over contexts of medium length where 256 rows
    // run meanwhile, of the formats whose walk goes by chunks (the others gain and lose 5 % there).  Otherwise a kernel of its own, which
    // merges too.  32 heads, a kernel of its own -> here, us (in launches back to back):
    //   CQ-8c8b   1 x 100 10.6 -> 7.6, 1 x 2000 10.5 -> 10.3, 1 x 3000 11.2 -> 11.2, 1 x 4096 10.9 -> 11.1, 4 x 4096 14.1 -> 14.0, 8 x 2000 13.9 ->
    //             11.8, 8 x 4096 16.3 -> 15.0, 8 x 16384 43.1 -> 41.4, 32 x 4096 45.5 -> 43.6
    //   CQ-4c8b   1 x 100 10.1 -> 8.0, 1 x 2000 12.1 -> 11.8, 1 x 4096 12.1 -> 12.4, 4 x 4096 16.4 -> 16.5, 8 x 4096 22.2 -> 21.1, 8 x 16384 68.0 -> 63.9
    //   CQ-2c8b   1 x 1000 15.1 -> 13.5, 1 x 2000 15.3 -> 15.3, 1 x 4096 15.6 -> 16.1, 8 x 2000 22.8 -> 21.6, 8 x 4096 34.7 -> 34.4, 8 x 16384 109.3 -> 110.6
    //   CQ-8c10b  1 x 1000 16.8 -> 15.3, 1 x 2000 16.2 -> 16.3, 1 x 4096 15.9 -> 16.9, 8 x 2000 24.2 -> 24.7, 16 x 2000 30.1 -> 28.8, 8 x 8192 40.4 -> 42.0,
    //             16 x 8192 58.3 -> 55.6
    const int rows = a.batch * a.n_q_heads;
    const bool by_chunks = a.f.b == 8 && a.f.gh <= 32;
    const bool short_rows = a.scores && a.n_q_heads == a.f.n_kv_heads && (a.t <= 2048 || (a.t <= 16384 && rows >= 256 && by_chunks));
    a.merge_counters = a.n_split > 1 && (!a.scores || short_rows) ? g_merge_counters.for_stream(stream, a.batch * a.n_q_heads) : nullptr;
    a.finish = short_rows && (a.n_split == 1 || a.merge_counters);
    const cq_status st = decode_takes_pairs(a) ? launch_decode_pair_view(a, stream)
                         : a.scores        ? launch_format<false, false, kScores>(a, stream)
                         : a.xk_new        ? launch_format<true, false, kWindow>(a, stream)
                                           : launch_format<false, false, kWindow>(a, stream);
    if (st == CQ_OK && a.scores && !a.finish) return launch_decode_weights(a, stream);
    if (st != CQ_OK || a.n_split == 1 || a.merge_counters || a.finish) return st;
    return launch_decode_merge(a, stream);
}

}  // namespace cq
