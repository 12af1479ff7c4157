// Eviction from a coded cache, for gfx950: which tokens of every (sequence, KV head) stay, and the caches and
// accumulators moved together.
//
// cq_select_tokens.  A stream's `keep` tokens are its first n_sink, its last n_recent and, between them, the heaviest,
// ties to the lowest index.  The weight of the last one that stays is found by its digits (a radix selection on the
// weights' order-preserving integers); what is above it stays, and of what equals it the first few.  Ranks come from
// counts in index order, so the list is ascending and a function of the weights alone.
//
// cq_compact_cache.  The token of rank r moves to position r.  A record's bytes are rotated by its token's position in
// the tile (slot s of token u holds group (s + u) mod Gh), so a move from u to u' rotates the record by u' - u bytes
// (10-bit codes: the word of high bits by twice as many bits).  A lane moves a token's record.
// Bound by memory.
#include "cq_decode_common.hpp"

namespace cq {
namespace {

// ---------------------------------------------------------------------------------- selection
constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kDigitBits = 11;                          // three digits: 11, 11, 10 bits
constexpr int kBins = 1 << kDigitBits;

// order-preserving: larger weights have larger keys, both zeros the same; what is no number ranks below every number
__device__ __forceinline__ unsigned weight_key(float w)
{
    const unsigned u = __float_as_uint(w + 0.f);
    if (w != w) return 0;
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// exclusive prefix sum over the workgroup's threads; *total: the sum
__device__ __forceinline__ unsigned block_prefix(unsigned v, unsigned* sums, int tid, unsigned* total)
{
    const int lane = tid & 63, wave = tid >> 6;
    unsigned x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned y = __shfl_up(x, d);
        x += lane >= d ? y : 0u;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        const unsigned s = sums[w];
        before += w < wave ? s : 0u;
        all += s;
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

__global__ __launch_bounds__(kSelectThreads) void select_tokens_kernel(SelectArgs a)
{
    __shared__ unsigned hist[kBins];
    __shared__ unsigned sums[kSelectWaves];
    __shared__ unsigned found[2];
    const int tid = threadIdx.x;
    const int stream = blockIdx.x, n = stream / a.n_kv_heads;
    int t_n = a.t;
    if (a.seq_lens) t_n = min(max(a.seq_lens[n], 0), a.t);
    int32_t* kept = a.kept + (size_t)stream * a.keep;
    if (stream % a.n_kv_heads == 0 && tid == 0) a.kept_lens[n] = min(t_n, a.keep);
    if (t_n <= a.keep) {
        for (int r = tid; r < a.keep; r += kSelectThreads) kept[r] = r < t_n ? r : -1;
        return;
    }
    for (int r = tid; r < a.n_sink; r += kSelectThreads) kept[r] = r;
    for (int r = tid; r < a.n_recent; r += kSelectThreads) kept[a.keep - a.n_recent + r] = t_n - a.n_recent + r;
    const float* w = a.weights + (size_t)stream * a.weights_stride + a.n_sink;
    const int len = t_n - a.n_sink - a.n_recent;            // the tokens between
    unsigned need = (unsigned)(a.keep - a.n_sink - a.n_recent);
    if (need == 0) return;
    // the key of the need-th largest, digit by digit
    unsigned prefix = 0, mask = 0;
#pragma unroll 1
    for (int shift = 21; shift >= 0; shift -= shift == 10 ? 10 : 11) {
        const int bins = shift == 0 ? kBins / 2 : kBins;
        for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < len; i += kSelectThreads) {
            const unsigned k = weight_key(w[i]);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        // thread i holds the bins 2 i, 2 i + 1 from the top; the bin in which `need` is reached
        const int hi = bins - 1 - 2 * tid;
        const unsigned c0 = hi >= 0 ? hist[hi] : 0u, c1 = hi >= 1 ? hist[hi - 1] : 0u;
        unsigned total;
        const unsigned above = block_prefix(c0 + c1, sums, tid, &total);
        if (above < need && above + c0 + c1 >= need) {
            const bool second = above + c0 < need;
            found[0] = (unsigned)(second ? hi - 1 : hi);
            found[1] = need - above - (second ? c0 : 0u);
        }
        __syncthreads();
        prefix |= found[0] << shift;
        mask |= (unsigned)(bins - 1) << shift;
        need = found[1];
        __syncthreads();
    }
    // ranks: those above the key, and the first `need` that equal it
    unsigned gt_base = 0, eq_base = 0;
    for (int i0 = 0; i0 < len; i0 += kSelectThreads) {
        const int i = i0 + tid;
        const unsigned k = i < len ? weight_key(w[i]) : 0u;
        const bool gt = i < len && k > prefix, eq = i < len && k == prefix;
        unsigned total;
        const unsigned at = block_prefix((gt ? 1u : 0u) | (eq ? 0x10000u : 0u), sums, tid, &total);
        const unsigned gts = gt_base + (at & 0xffffu), eqs = eq_base + (at >> 16);
        if (gt || (eq && eqs < need)) kept[a.n_sink + gts + min(eqs, need)] = a.n_sink + i;
        gt_base += total & 0xffffu;
        eq_base += total >> 16;
    }
}

// ---------------------------------------------------------------------------------- moving
constexpr int kMoveThreads = 256;

// out byte i = in byte (i + by) mod 4 W
template <int W>
__device__ __forceinline__ void rotate_bytes(unsigned (&w)[W], unsigned by)
{
#pragma unroll
    for (int d = 1; d < W; d *= 2) {
        const bool on = (by >> 2) & (unsigned)d;
        unsigned x[W];
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = on ? w[(i + d) % W] : w[i];
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = x[i];
    }
    const unsigned first = w[0];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = __builtin_amdgcn_alignbyte(i + 1 < W ? w[i + 1] : first, w[i], by & 3u);
}

// a token's record: Gh low bytes in 16-byte pieces, and (b = 10) the word of high bits
template <int GH, int B>
struct Record {
    unsigned w[GH / 4];
    unsigned hi;
    __device__ __forceinline__ void load(const uint8_t* tile, int u)
    {
#pragma unroll
        for (int p = 0; p < GH / 16; ++p) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(tile + p * 1024 + u * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * p + i] = x[i];
        }
        if constexpr (B == 10) hi = *reinterpret_cast<const unsigned*>(tile + kTileTokens * GH + u * 4);
    }
    __device__ __forceinline__ void store(uint8_t* tile, int u) const
    {
#pragma unroll
        for (int p = 0; p < GH / 16; ++p)
            *reinterpret_cast<u32x4*>(tile + p * 1024 + u * 16) = u32x4{w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]};
        if constexpr (B == 10) *reinterpret_cast<unsigned*>(tile + kTileTokens * GH + u * 4) = hi;
    }
    __device__ __forceinline__ void move(int from, int to)
    {
        const unsigned by = (unsigned)(to - from) & (unsigned)(GH - 1);
        rotate_bytes(w, by);
        if constexpr (B == 10) hi = __builtin_amdgcn_alignbit(hi, hi, 2 * by);
    }
};

// A wavefront moves a tile of one stream of one cache.  GATHER: from a token's old position to its new one (in the caches,
// or in the workspace where the caches' own places are still to be read); else from the workspace to the caches.
template <int GH, int B, bool GATHER>
__global__ __launch_bounds__(kMoveThreads) void move_tokens_kernel(CompactArgs a, int tiles, int64_t items)
{
    constexpr int TILE = kTileTokens * GH * B / 8;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * (kMoveThreads / 64) + (threadIdx.x >> 6);
    if (item >= items) return;
    const int which = (int)(item & 1);
    const int64_t rest = item >> 1;
    const int tile = (int)(rest % tiles), stream = (int)(rest / tiles);
    const int n = stream / a.n_kv_heads, h = stream % a.n_kv_heads;
    const int count = min(max(a.kept_lens[n], 0), a.keep);
    const int r = tile * kTileTokens + lane;
    uint8_t* const work = a.work ? a.work + ((size_t)item) * TILE : nullptr;
    float* const work_weights = a.work_weights ? a.work_weights + (size_t)stream * a.keep : nullptr;
    if (r < count) {
        Record<GH, B> rec;
        uint8_t* const out = work && GATHER ? work : a.out[which] + a.map_out.tile_index(n, h, tile) * TILE;
        if constexpr (GATHER) {
            const int from = min(max(a.kept[(size_t)stream * a.keep + r], 0), a.t - 1);
            rec.load(a.in[which] + a.map_in.tile_index(n, h, from / kTileTokens) * TILE, from % kTileTokens);
            rec.move(from % kTileTokens, lane);
            if (which == 0 && a.weights) {
                const float x = a.weights[(size_t)stream * a.weights_stride + from];
                if (work) work_weights[r] = x;
                else a.weights_out[(size_t)stream * a.weights_out_stride + r] = x;
            }
        } else {
            rec.load(work, lane);
            if (which == 0 && a.weights) a.weights_out[(size_t)stream * a.weights_out_stride + r] = work_weights[r];
        }
        rec.store(out, lane);
    }
}

// accumulators behind the tokens that stay: zero, up to `end`
__global__ __launch_bounds__(kMoveThreads) void clear_weights_kernel(CompactArgs a, int end)
{
    const int stream = blockIdx.y, n = stream / a.n_kv_heads;
    const int count = min(max(a.kept_lens[n], 0), a.keep);
    const int i = blockIdx.x * kMoveThreads + threadIdx.x;
    if (i >= count && i < end) a.weights_out[(size_t)stream * a.weights_out_stride + i] = 0.f;
}

template <int GH, int B>
cq_status launch_move(const CompactArgs& a, hipStream_t stream)
{
    const int tiles = (a.keep + kTileTokens - 1) / kTileTokens;
    const int64_t items = (int64_t)2 * a.batch * a.n_kv_heads * tiles, wgs = (items + kMoveThreads / 64 - 1) / (kMoveThreads / 64);
    if (wgs > 0x7fffffffLL) return CQ_ERR_INVALID_ARG;
    hipLaunchKernelGGL((move_tokens_kernel<GH, B, true>), dim3((unsigned)wgs), dim3(kMoveThreads), 0, stream, a, tiles, items);
    if (hipGetLastError() != hipSuccess) return CQ_ERR_HIP;
    if (a.work) {
        hipLaunchKernelGGL((move_tokens_kernel<GH, B, false>), dim3((unsigned)wgs), dim3(kMoveThreads), 0, stream, a, tiles, items);
        if (hipGetLastError() != hipSuccess) return CQ_ERR_HIP;
    }
    if (!a.weights) return CQ_OK;
    const int end = a.t < a.t_cap_out ? a.t : a.t_cap_out;
    const int streams = a.batch * a.n_kv_heads;
    if (streams > 65535) return CQ_ERR_INVALID_ARG;
    hipLaunchKernelGGL(clear_weights_kernel, dim3((unsigned)((end + kMoveThreads - 1) / kMoveThreads), (unsigned)streams), dim3(kMoveThreads), 0, stream, a, end);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

}  // namespace

cq_status launch_select_tokens(const SelectArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL(select_tokens_kernel, dim3((unsigned)(a.batch * a.n_kv_heads)), dim3(kSelectThreads), 0, stream, a);
    return hipGetLastError() == hipSuccess ? CQ_OK : CQ_ERR_HIP;
}

cq_status launch_compact(const CompactArgs& a, const Derived& f, hipStream_t stream)
{
    if (f.b == 10) return launch_move<16, 10>(a, stream);
    if (f.gh == 16) return launch_move<16, 8>(a, stream);
    if (f.gh == 32) return launch_move<32, 8>(a, stream);
    if (f.gh == 64) return launch_move<64, 8>(a, stream);
    return CQ_ERR_UNSUPPORTED;
}

}  // namespace cq
