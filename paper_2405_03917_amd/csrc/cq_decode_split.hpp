// Device code shared by the two kernels of decode attention over keys as stored (cq_decode.hip: a query head per
// workgroup; cq_decode_pair.hip: two): partials and their merge, the new token's record, a tile's request.
#pragma once

#include "cq_decode_common.hpp"

namespace cq {
namespace {

constexpr int kDecodeThreads = 512;
constexpr int kDecodeWaves = kDecodeThreads / 64;
// tiles per wavefront and chunk (= score registers per lane): b = 8: 16, and 8 for splits that fit;
// b = 10: 32 (one chunk must hold the longest split, 16384 tokens), and 16 for splits that fit
constexpr int kChunkTiles8 = 16;
constexpr int kChunkTiles10 = 32;

// What a call sees of a sequence, and what it returns besides the output.
enum View : int {
    kWhole = 0,         // every token
    kWindow = 1,        // the last `window` tokens and the first n_sink
    kScores = 2,        // every token, and the scores go to memory
};

// The tiles of a sequence that a call walks, numbered without gaps: of a window, the sinks' tiles in front of it (`head`
// of them), then its own, `skip` tiles further on in the cache.  Every tile of the view holds a token that is seen.
template <int VIEW>
struct Seen {
    int n_tiles;
    __device__ __forceinline__ Seen() = default;
    __device__ __forceinline__ Seen(const DecodeArgs&, int t_n) : n_tiles((t_n + kTileTokens - 1) / kTileTokens) {}
    __device__ __forceinline__ int tile(int i) const { return i; }
    __device__ __forceinline__ bool edge(int i) const { return i == n_tiles - 1; }      // tiles that hold tokens not seen
    __device__ __forceinline__ bool token(int tok, int t_n) const { return tok < t_n; }
};
template <>
struct Seen<kWindow> {
    int n_tiles, head, skip, first, n_sink;             // first: the window's first token
    __device__ __forceinline__ Seen() = default;
    __host__ __device__ __forceinline__ Seen(const DecodeViewArgs& a, int t_n)
    {
        n_sink = a.n_sink;
        first = max(0, t_n - a.window);
        const int at = first / kTileTokens;
        head = min((n_sink + kTileTokens - 1) / kTileTokens, at);
        skip = at - head;
        n_tiles = (t_n + kTileTokens - 1) / kTileTokens - skip;
    }
    __host__ __device__ __forceinline__ int tile(int i) const { return i < head ? i : i + skip; }
    __host__ __device__ __forceinline__ bool edge(int i) const { return i == n_tiles - 1 || i == head || i == head - 1; }
    __host__ __device__ __forceinline__ bool token(int tok, int t_n) const { return tok < t_n && (tok >= first || tok < n_sink); }
};

// LayerPtrs as the kernel reads it.  A pointer read from memory could point anywhere (LDS,
// scratch) as far as the compiler knows, and every access through it would be a flat instruction,
// which waits on the LDS counter and the memory counter at once; the table's pointers are
// therefore declared as what they are, pointers into global memory.
#define CQ_GLOBAL __attribute__((address_space(1)))
struct LayerPtrsGlobal {
    CQ_GLOBAL const uint16_t* q;
    CQ_GLOBAL const uint16_t* xk_new;
    CQ_GLOBAL const uint16_t* xv_new;
    CQ_GLOBAL uint8_t* k_codes;
    CQ_GLOBAL uint8_t* v_codes;
    CQ_GLOBAL const uint16_t* k_centroids;
    CQ_GLOBAL const uint16_t* v_centroids;
    CQ_GLOBAL uint16_t* out;
};
#undef CQ_GLOBAL
static_assert(sizeof(LayerPtrsGlobal) == sizeof(LayerPtrs), "same record");

// Merge the partials of all splits of one (sequence, query head): one pass with a running
// maximum (the usual rescaling), so that no load waits for a value computed from another and
// the loads of all splits go out together; then one rounding to fp16.  A split beyond its
// sequence left m = -inf, l = 0, o = 0 and gets weight 0.  DEVICE_LOADS: the partials were
// written by other workgroups of the running kernel: read them with device-scope loads.
template <bool DEVICE_LOADS>
__device__ __forceinline__ float partial_load(const float* p)
{
    if constexpr (DEVICE_LOADS) return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else return *p;
}
template <bool DEVICE_LOADS>
__device__ __forceinline__ void merge_splits(const float* p, int n_split, int head_dim, uint16_t* out, int tid, int nt)
{
    const int stride = head_dim + kPartialHeader;
    for (int i = tid; i < head_dim; i += nt) {
        float m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll 4
        for (int s = 0; s < n_split; ++s) {
            const float ms = partial_load<DEVICE_LOADS>(p + s * stride), ls = partial_load<DEVICE_LOADS>(p + s * stride + 1),
                        os = partial_load<DEVICE_LOADS>(p + s * stride + kPartialHeader + i);
            const float m_new = fmaxf(m, ms);
            const float m_safe = m_new == -INFINITY ? 0.f : m_new;
            const float keep = __builtin_amdgcn_exp2f(m - m_safe), w = __builtin_amdgcn_exp2f(ms - m_safe);
            l = __builtin_fmaf(l, keep, ls * w);
            o = __builtin_fmaf(o, keep, os * w);
            m = m_new;
        }
        const _Float16 h = (_Float16)(o / l);
        out[i] = __builtin_bit_cast(uint16_t, h);
    }
}
// (device-scope store: written through to where every workgroup's device-scope loads find it)
__device__ __forceinline__ void partial_store(float* p, float v)
{
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// kScores: the score of a row's token to memory (where other workgroups of the running kernel read it, device-scope).
template <int VIEW, class Args>
__device__ __forceinline__ void keep_score(const Args& a, size_t row, int tok, float s)
{
    if constexpr (VIEW == kScores) {
        float* const at = a.scores + row * a.score_stride + tok;
        if (a.finish) partial_store(at, s);
        else *at = s;
    }
}
// kScores: a split's reference and sum.  (The sum of the probabilities in fixed point, by which the output is divided, is no
// substitute: equal probabilities of a long context are all rounded the same way, 1e-4 of their sum at 131072 tokens.)
template <int VIEW, class Args>
__device__ __forceinline__ void keep_stats(const Args& a, size_t row, int split, float m, float l)
{
    if constexpr (VIEW == kScores) {
        float* const at = reinterpret_cast<float*>(a.stats + row * a.n_split + split);
        partial_store(at, m);
        partial_store(at + 1, l);
    }
}
// A row's softmax reference and the reciprocal of its sum, from those of its splits (by a wavefront).
template <bool DEVICE_LOADS>
__device__ __forceinline__ float2 row_stats(const DecodeViewArgs& a, size_t row, int lane)
{
    const float* p = reinterpret_cast<const float*>(a.stats + row * a.n_split);
    float m = -INFINITY;
    for (int s = lane; s < a.n_split; s += 64) m = fmaxf(m, partial_load<DEVICE_LOADS>(p + 2 * s));
    m = wave_max(m);
    float l = 0.f;
    for (int s = lane; s < a.n_split; s += 64)
        l = __builtin_fmaf(partial_load<DEVICE_LOADS>(p + 2 * s + 1), __builtin_amdgcn_exp2f(partial_load<DEVICE_LOADS>(p + 2 * s) - m), l);
    l = wave_sum(l);
    return make_float2(m, 1.f / l);
}
// The accumulators of a KV head with one query head, by a workgroup, once all of the row's scores and statistics are written.
template <int VIEW, class Args>
__device__ __forceinline__ void finish_weights(const Args& a, size_t row, int t_n, int tid, int nt)
{
    if constexpr (VIEW == kScores) {
        constexpr int N = 8;                                // tokens of a thread that are requested together
        const float* s = a.scores + row * a.score_stride;
        float* acc = a.weights + row * a.weights_stride;
        float2 st;
        for (int base = 0; base < t_n; base += N * nt) {       // (uniform: row_stats exchanges between all lanes)
            float score[N], old[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int tok = base + tid + k * nt;
                score[k] = tok < t_n ? partial_load<true>(s + tok) : 0.f;
                old[k] = a.decay != 0.f && tok < t_n ? acc[tok] : 0.f;
            }
            if (base == 0) st = row_stats<true>(a, row, tid & 63);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int tok = base + tid + k * nt;
                const float w = __builtin_fmaf(__builtin_amdgcn_exp2f(score[k] - st.x), st.y, 0.f);
                if (tok < t_n) acc[tok] = __builtin_fmaf(a.decay, old[k], w);
            }
        }
    }
}

// The last split of a (sequence, query head) to finish merges them all.  Partials are written with device-scope
// stores (write-through) and the merging workgroup reads them with device-scope loads, so
// no cache has to be written back or invalidated as a whole (a device-scope release fence
// per workgroup, which writes the whole L2 back, cost 50 us on a 90 us launch).  Order:
// every wavefront waits for its stores (a barrier does not, __syncthreads() neither), then all meet at the
// barrier, then one thread counts the workgroup in; the workgroup that counts the last split (true) takes the counter
// back to zero for the next call.
template <int D>
__device__ __forceinline__ bool counted_last(const DecodeArgs& a, const float* part, unsigned* flag, int tid)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        const size_t row = (size_t)(part - a.partials) / ((size_t)(D + kPartialHeader) * a.n_split);
        const unsigned arrived = __hip_atomic_fetch_add(a.merge_counters + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = arrived == (unsigned)a.n_split - 1u;
        if (last) __hip_atomic_store(a.merge_counters + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = last;
    }
    __syncthreads();
    return *flag != 0u;
}

// Fused step: words of LDS from the keys on.  The 2 Gh 64-bit minima; the new token's fixed-point weight, one per query
// head of the workgroup, in 16 bytes; the record of its key codes (NewTokenRecord), read 16 bytes at a time.
template <int GH, int B>
struct NewTokenWords {
    static constexpr int WEIGHT = 2 * 2 * GH;
    static constexpr int RECORD = WEIGHT + 4;
    static constexpr int END = RECORD + GH / 4 + (B == 10 ? 1 : 0);
};

// Fused step: the key codes of the new token as the cache layout would hold them (slot s of token
// u carries group (s + u) mod Gh), from keys[g] = group g's (distance, index) minimum.  Built in LDS
// by the one wavefront whose walk meets the token's tile, before its walk starts (lane i builds word
// i); when the walk reaches the tile, lane u's codes are replaced by the record.
template <int GH, int B>
struct NewTokenRecord {
    unsigned* rec;                      // [GH / 4] words of low bytes, then (b = 10) the word of high bits
    __device__ __forceinline__ void build(const unsigned long long* keys, int u_new, int lane) const
    {
        unsigned x = 0, h = 0;
        if (lane < GH / 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int s = 4 * lane + k;
                const unsigned code = (unsigned)(keys[(s + u_new) & (GH - 1)] & 0xffffffffu);
                x |= (code & 0xffu) << (8 * k);
                if constexpr (B == 10) h |= (code >> 8) << (2 * s);
            }
            rec[lane] = x;
        }
        if constexpr (B == 10) {
            static_assert(B != 10 || GH == 16, "four lanes hold the high bits");
            h |= __shfl_xor(h, 1);
            h |= __shfl_xor(h, 2);
            if (lane == 0) rec[GH / 4] = h;
        }
    }
    __device__ __forceinline__ void patch(Tile<GH, B>& w, int u_new, int lane) const
    {
        const bool mine = lane == u_new;
#pragma unroll
        for (int pl = 0; pl < GH / 16; ++pl) {
            const uint4 r = *reinterpret_cast<const uint4*>(rec + 4 * pl);
            u32x4 q = w.lo[pl];
            q.x = mine ? r.x : q.x;
            q.y = mine ? r.y : q.y;
            q.z = mine ? r.z : q.z;
            q.w = mine ? r.w : q.w;
            w.lo[pl] = q;
        }
        if constexpr (B == 10) w.hi = mine ? rec[GH / 4] : w.hi;
    }
};

// One 64-token tile through a buffer descriptor of its own: `tile` is wave-uniform; a tile that
// does not exist gets a descriptor of size zero, for which the hardware returns zeros without
// touching memory.  Every request of the walk is therefore issued unconditionally, and the
// number of loads in flight at any point of the (unrolled) walk is a compile-time constant.
template <int GH, int B>
__device__ __forceinline__ Tile<GH, B> load_tile_desc(const uint8_t* tile, bool exists, int lane)
{
    constexpr int TB = kTileTokens * GH * B / 8;
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(tile), 0, exists ? TB : 0, 0x00020000);
    Tile<GH, B> w;
    const unsigned off = 16u * (unsigned)lane;
#pragma unroll
    for (int pl = 0; pl < GH / 16; ++pl)
        w.lo[pl] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + 1024u * pl, 0, 2));
    if constexpr (B == 10)
        w.hi = __builtin_amdgcn_raw_buffer_load_b32(rsrc, 4u * (unsigned)lane + (unsigned)(kTileTokens * GH), 0, 2);
    else
        w.hi = 0;
    return w;
}

}  // namespace
}  // namespace cq
